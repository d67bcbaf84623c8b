// ffn.hip -- the gated feed-forward block in 16-bit types, forward and
// backward, as three matrix products on the matrix cores:
//   forward   g = x Wg^T, u = x Wu^T, h = act(g) u      (one launch)
//   gradients dg = gh u act'(g), du = gh act(g)         (elementwise)
//             gx = dg Wg + du Wu;  gWg = dg^T x, gWu = du^T x
// One kernel template computes C[r][c] = sum_k R(r, k) Q(c, k) over tiles of
// 128 x 128: operands whose k runs along their rows ("row form": x, W in the
// forward, dg/du in gx) are read from LDS as 16 bytes per lane, operands whose
// k runs down their columns ("column form": W in gx, all of gW) through the
// transposing LDS reads.
#include "dense_rows.h"

#include "qconv_internal.h"

namespace qc {

namespace {

constexpr int KSTEP = 64;  // products per LDS stage

typedef __attribute__((address_space(3))) void* lds_ptr;

// Row form: value (r, k) at p[r * ld + k]; column form: at p[k * ld + r].
struct Operand {
  const uint16_t* p;
  int64_t ld;
};

enum GemmOut { OUT_GATED = 0, OUT_PLAIN = 1 };

struct GemmArgs {
  Operand r[2], c[2];  // by segment (the sums of gx run over two operand pairs) or by half (gW's two outputs)
  int rows, cols, k;   // C's extent (of one half) and the products of one segment
  int segments;        // 1 or 2
  int halves;          // 2: a second C from r[1] with the same c[0]
  int tiles_r, tiles_c;
  void* out[2];
  int64_t ld_out;
  int wide_out;  // rows of out (and of pre) start at 8-byte addresses
  float* pre;    // OUT_GATED: [rows][2][ld_pre] or NULL
  int ld_pre;
  int act;
};

// LDS holds chunks of 16 bytes.  Row form: rows of 64 products (8 chunks)
// with the chunk index xored by the row, so that the 16 rows of a fragment
// read lie in different banks.  Column form: one LDS row per product, of ROWS
// values; a transposing read touches 4 of them at one place, and the lanes
// beside it 4 more 8 rows below, which the xor spreads over the banks.
__device__ __forceinline__ int swz_row(int r) { return r & 7; }
__device__ __forceinline__ int swz_col(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) << 1; }

// The tile of one operand: ROWS rows (or columns) of C by KSTEP products,
// staged by NT threads, CH chunks each.
//
// ALIGNED: every row of the operand starts at a 16-byte address and the rows'
// length (k in row form) is a multiple of 8, so each chunk is one 16-byte load
// straight into LDS; chunks past the ends get an offset past the buffer's
// range, which loads zeros.  Otherwise chunks pass through registers, and the
// ones that cross an end are read value by value.
//
// PAIR: the gated forward's columns.  64 columns of the tile are 32 gate rows
// and the 32 up rows of the same hidden features, so that one lane ends up
// with both sums.
template <int ROWS, int NT, bool COL, bool ALIGNED, bool PAIR>
struct Stage {
  static constexpr int CH = ROWS * KSTEP / 8 / NT;
  const uint16_t *p, *p2;  // the tile's first value, product 0
  int64_t ld;
  int rows;  // rows of the operand from the tile's first (gate rows for PAIR)
  typedef std::conditional_t<ALIGNED, uint32_t, int64_t> Off;
  static constexpr Off OUTSIDE = ALIGNED ? (Off)0x80000000u : (Off)-1;
  Off off[CH];      // byte offset of each chunk from p, or OUTSIDE
  int at[CH];       // its first product (row form) or its product (column form)
  v4u reg[ALIGNED ? 1 : CH];

  __device__ __forceinline__ static int chunk(int j) { return (int)threadIdx.x + j * NT; }

  __device__ __forceinline__ void init(const Operand& o, const Operand& o2, int64_t r0, int64_t all) {
    p = o.p + (COL ? r0 : r0 * o.ld);
    p2 = PAIR ? o2.p + r0 * o.ld : nullptr;
    ld = o.ld;
    rows = (int)(all - r0 < 0x7fffff00 ? all - r0 : 0x7fffff00);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = chunk(j);
      if constexpr (COL) {
        const int k = c / (ROWS / 8), r = ((c % (ROWS / 8)) ^ swz_col(k)) * 8;
        at[j] = k;
        off[j] = r < rows ? (Off)(k * ld + r) * 2 : OUTSIDE;
      } else {
        const int t = c / 8, k = ((c % 8) ^ swz_row(t)) * 8;
        const int r = PAIR ? (t / 64) * 32 + t % 32 : t;
        at[j] = k;
        off[j] = r < rows ? (Off)(r * ld + k) * 2 : OUTSIDE;
      }
    }
  }

  // Products [k0, k0 + KSTEP) of `k`, into (or on the way to) the stage at lds.
  __device__ __forceinline__ void load(v4u* lds, int k0, int k) {
    const int left = k - k0;
    const uint16_t* b = p + (COL ? k0 * ld : (int64_t)k0);
    if constexpr (ALIGNED) {
      const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)b, (short)0, 0x7fffffff, 0x00020000);
      const auto rs2 = __builtin_amdgcn_make_buffer_rsrc((void*)(PAIR ? p2 + k0 : b), (short)0, 0x7fffffff, 0x00020000);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63) + j * NT;  // the wave's first chunk
        const uint32_t o = at[j] < left ? off[j] : OUTSIDE;
        // a wave's 64 chunks are 8 rows, so all of them gate or all of them up
        if (PAIR && ((w / 8) & 32))
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rs2, (lds_ptr)(lds + w), 16, o, 0, 0, 0);
        else
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + w), 16, o, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const uint16_t* q = PAIR && ((chunk(j) / 8) & 32) ? p2 + k0 : b;
        const int c = chunk(j);
        const int n = COL ? rows - ((c % (ROWS / 8)) ^ swz_col(c / (ROWS / 8))) * 8 : left - at[j];
        const bool in = off[j] != OUTSIDE && at[j] < left;
        reg[j] = load8_first(in ? (const uint16_t*)((const char*)q + off[j]) : q, in ? n : 0);
      }
    }
  }
  // The rest of load(), once the stage's last readers are done.
  __device__ __forceinline__ void store(v4u* lds) {
    if constexpr (!ALIGNED) {
#pragma unroll
      for (int j = 0; j < CH; ++j) lds[chunk(j)] = reg[j];
    }
  }
};

// The 8 products [s * 32 + (lane / 16) * 8, +8) of tile row r0 + lane % 16.
template <int ROWS, bool COL>
__device__ __forceinline__ v4u fragment(const v4u* lds, int r0, int s) {
  const int lane = threadIdx.x & 63;
  if constexpr (!COL) {
    const int r = r0 + (lane & 15);
    return lds[r * 8 + ((s * 4 + (lane >> 4)) ^ swz_row(r))];
  } else {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s* lp;
    v2u h[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // 16 lanes read 4 LDS rows of 16 values and get them transposed: lane i
      // holds column i of the 4
      const int k = s * 32 + (lane >> 4) * 8 + j * 4 + ((lane & 15) >> 2);
      const int c = r0 / 8 + ((lane & 3) >> 1);
      const char* at = (const char*)(lds + k * (ROWS / 8) + (c ^ swz_col(k))) + (lane & 1) * 8;
      h[j] = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)at));
    }
    return v4u{h[0][0], h[0][1], h[1][0], h[1][1]};
  }
}

// Four values of one row, columns c..c + 3 of `cols`.
template <class T>
__device__ __forceinline__ void put4(void* out, int64_t row, int64_t c, int64_t cols, bool wide, const float v[4]) {
  uint16_t* p = (uint16_t*)out + row + c;
  uint16_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = T::down(v[e]);
  if (wide && c + 4 <= cols) {
    *(v2u*)p = v2u{b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < cols) p[e] = b[e];
  }
}

// A block computes a BR x BC tile of C with waves of (BR / 2) x 64 each.
// Two LDS stages: while the waves multiply one, the next is loaded.
template <class T, bool RCOL, bool CCOL, int OUT, int BR, int BC, bool ALIGNED>
__global__ __launch_bounds__(BC / 64 * 128) void ffn_gemm_kernel(GemmArgs a) {
  constexpr int NT = BC / 64 * 128, NR = BR / 32, PAIR = OUT == OUT_GATED;
  constexpr int LR = BR * KSTEP / 8, LC = BC * KSTEP / 8;
  __shared__ v4u lds[2][LR + LC];
  // Workgroups go to the 8 dies in turn; each die gets a run of tiles that
  // share operands in its L2: 8 tile rows at a time, column after column.
  const uint32_t all = gridDim.x, die = blockIdx.x & 7;
  const uint32_t tile = die * (all / 8) + (die < all % 8 ? die : all % 8) + blockIdx.x / 8;
  const uint32_t trs = a.tiles_r * a.halves, group = 8 * a.tiles_c;
  const uint32_t first = tile / group * 8, some = trs - first < 8 ? trs - first : 8;
  const uint32_t tr = first + tile % group % some, tc = tile % group / some;
  const int half = tr >= (uint32_t)a.tiles_r;
  const int64_t r0 = (int64_t)(tr - half * a.tiles_r) * BR;
  const int64_t c0 = (int64_t)tc * (PAIR ? BC / 2 : BC);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int wr = (wave & 1) * (BR / 2), wc = (wave >> 1) * 64;
  v4f acc[4][NR];  // [column group][row group]: lane holds row lane % 16, columns (lane / 16) * 4 + 0..3
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NR; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  Stage<BR, NT, RCOL, ALIGNED, false> sr;
  Stage<BC, NT, CCOL, ALIGNED, PAIR> sc;
  const int steps = ceil_div(a.k, KSTEP), total = steps * a.segments;
  sr.init(a.r[half], a.r[half], r0, a.rows);
  sc.init(a.c[0], a.c[1], c0, a.cols);
  if (total > 0) {
    sr.load(lds[0], 0, a.k);
    sc.load(lds[0] + LR, 0, a.k);
    sr.store(lds[0]);
    sc.store(lds[0] + LR);
  }
  int k0 = 0;
  for (int step = 0; step < total; ++step) {
    const int b = step & 1;
    if constexpr (ALIGNED) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads into LDS are not waited for elsewhere
    lds_barrier();
    k0 += KSTEP;
    if (step + 1 == steps && a.segments == 2) {
      sr.init(a.r[1], a.r[1], r0, a.rows);
      sc.init(a.c[1], a.c[1], c0, a.cols);
      k0 = 0;
    }
    if (step + 1 < total) {
      sr.load(lds[b ^ 1], k0, a.k);
      sc.load(lds[b ^ 1] + LR, k0, a.k);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      v4u fr[NR], fc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) fc[i] = fragment<BC, CCOL>(lds[b] + LR, wc + i * 16, s);
#pragma unroll
      for (int i = 0; i < NR; ++i) fr[i] = fragment<BR, RCOL>(lds[b], wr + i * 16, s);
#pragma unroll
      for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = T::mfma(fc[i], fr[j], acc[i][j]);
    }
    if (step + 1 < total) {
      sr.store(lds[b ^ 1]);
      sc.store(lds[b ^ 1] + LR);
    }
  }
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int64_t r = r0 + wr + j * 16 + (lane & 15);
    if (r >= a.rows) continue;
    if constexpr (PAIR) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t f = c0 + wc / 2 + i * 16 + (lane >> 4) * 4;
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = act_value(a.act, acc[i][j][e]) * acc[i + 2][j][e];
        put4<T>(a.out[0], r * a.ld_out, f, a.cols, a.wide_out, h);
        if (a.pre) {
          float* g = a.pre + r * 2 * a.ld_pre + f;
          if (f + 4 <= a.cols) {
            *(v4f*)g = acc[i][j];
            *(v4f*)(g + a.ld_pre) = acc[i + 2][j];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (f + e < a.cols) {
                g[e] = acc[i][j][e];
                g[a.ld_pre + e] = acc[i + 2][j][e];
              }
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t c = c0 + wc + i * 16 + (lane >> 4) * 4;
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        put4<T>(a.out[half], r * a.ld_out, c, a.cols, a.wide_out, v);
      }
    }
  }
}

// dg and du of four hidden features per thread, into [m][2][fp] with the
// columns past f zero (gx's products run over all fp of them).
template <class T, int ACT>
__global__ __launch_bounds__(256) void ffn_slopes_kernel(const float* __restrict__ pre, const uint16_t* __restrict__ gh,
                                                         int64_t ld_h, int m, int f, int fp,
                                                         uint16_t* __restrict__ d) {
  const int64_t n = (int64_t)m * (fp / 4);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / (fp / 4);
    const int c = (int)(i % (fp / 4)) * 4;
    const v4f g = *(const v4f*)(pre + r * 2 * fp + c), u = *(const v4f*)(pre + (r * 2 + 1) * fp + c);
    uint16_t dg[4], du[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = c + e < f;
      const float gr = in ? T::up(gh[r * ld_h + c + e]) : 0.0f;
      dg[e] = in ? T::down(gr * u[e] * act_slope<ACT>(g[e])) : (uint16_t)0;
      du[e] = in ? T::down(gr * act_value<ACT>(g[e])) : (uint16_t)0;
    }
    *(v2u*)(d + r * 2 * fp + c) = v2u{dg[0] | (uint32_t)dg[1] << 16, dg[2] | (uint32_t)dg[3] << 16};
    *(v2u*)(d + (r * 2 + 1) * fp + c) = v2u{du[0] | (uint32_t)du[1] << 16, du[2] | (uint32_t)du[3] << 16};
  }
}

template <class T, bool RCOL, bool CCOL, int OUT, int B, bool ALIGNED>
int run_tiles(GemmArgs& a, hipStream_t s) {
  a.tiles_r = ceil_div(a.rows, B);
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? B / 2 : B);
  const int64_t blocks = (int64_t)a.tiles_r * a.tiles_c * a.halves;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  ffn_gemm_kernel<T, RCOL, CCOL, OUT, B, B, ALIGNED><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a);
  return hip_status();
}

// Every row of the operand starts at a 16-byte address, and a tile's offsets
// stay below 2^31 bytes.
bool aligned_rows(const Operand& o) { return ((uintptr_t)o.p & 15) == 0 && o.ld % 8 == 0 && o.ld < (1 << 21); }

template <class T, bool RCOL, bool CCOL, int OUT>
int run_gemm_t(GemmArgs& a, bool aligned, hipStream_t s) {
  if (!aligned) return run_tiles<T, RCOL, CCOL, OUT, 128, false>(a, s);
  const int64_t big = (int64_t)ceil_div(a.rows, 256) * ceil_div(a.cols, OUT == OUT_GATED ? 128 : 256) * a.halves;
  if (big >= 256) return run_tiles<T, RCOL, CCOL, OUT, 256, true>(a, s);
  return run_tiles<T, RCOL, CCOL, OUT, 128, true>(a, s);
}

template <bool RCOL, bool CCOL, int OUT>
int run_gemm(int dtype, GemmArgs& a, bool aligned, hipStream_t s) {
  a.wide_out = a.ld_out % 4 == 0 && ((uintptr_t)a.out[0] & 7) == 0 && ((uintptr_t)a.out[1] & 7) == 0;
  return dtype == QCONV_F16 ? run_gemm_t<F16, RCOL, CCOL, OUT>(a, aligned, s)
                            : run_gemm_t<BF16, RCOL, CCOL, OUT>(a, aligned, s);
}

template <class T>
int run_slopes(const qconv_ffn_desc& d, const float* pre, const void* gh, int fp, uint16_t* out, hipStream_t s) {
  const int64_t n = (int64_t)d.m * (fp / 4);
  const unsigned grid = (unsigned)(n < (1 << 23) ? (n + 255) / 256 : 1 << 15);
  const uint16_t* g = (const uint16_t*)gh;
  if (d.act == QCONV_ACT_SILU)
    ffn_slopes_kernel<T, QCONV_ACT_SILU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  else if (d.act == QCONV_ACT_GELU)
    ffn_slopes_kernel<T, QCONV_ACT_GELU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  else
    ffn_slopes_kernel<T, QCONV_ACT_RELU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  return hip_status();
}

}  // namespace

int launch_ffn_forward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, void* h, float* pre,
                       hipStream_t s) {
  if (d.m == 0) return QCONV_OK;
  if (d.m <= 64) {
    RowsArgs r = {};
    r.x = (const uint16_t*)x;
    r.ld_x = d.ld_x;
    r.ld_w = d.ld_w;
    r.ld_y = d.ld_h;
    r.w[0] = wg;
    r.w[1] = wu;
    r.y = (uint16_t*)h;
    r.pre = pre;
    r.ld_pre = (int)round_up(d.f, 8);
    r.m = d.m;
    r.n = d.f;
    r.k = d.k;
    r.act = d.act;
    return d.dtype == QCONV_F16 ? run_dense_rows<F16, Dense16, 2>(r, s) : run_dense_rows<BF16, Dense16, 2>(r, s);
  }
  GemmArgs a = {};
  a.r[0] = {(const uint16_t*)x, d.ld_x};
  a.c[0] = {(const uint16_t*)wg, d.ld_w};
  a.c[1] = {(const uint16_t*)wu, d.ld_w};
  a.rows = d.m;
  a.cols = d.f;
  a.k = d.k;
  a.segments = a.halves = 1;
  a.out[0] = h;
  a.ld_out = d.ld_h;
  a.pre = pre;
  a.ld_pre = (int)round_up(d.f, 8);
  a.act = d.act;
  const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && aligned_rows(a.c[1]) && d.k % 8 == 0;
  return run_gemm<false, false, OUT_GATED>(d.dtype, a, aligned, s);
}

size_t ffn_backward_bytes(const qconv_ffn_desc& d) { return (size_t)d.m * 2 * round_up(d.f, 8) * 2; }

int launch_ffn_backward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, const float* pre,
                        const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s) {
  const int fp = (int)round_up(d.f, 8);
  uint16_t* dgu = (uint16_t*)ws;
  int rc = QCONV_OK;
  if (d.m > 0)
    rc = d.dtype == QCONV_F16 ? run_slopes<F16>(d, pre, gh, fp, dgu, s) : run_slopes<BF16>(d, pre, gh, fp, dgu, s);
  if (rc == QCONV_OK && gx && d.m > 0) {
    GemmArgs a = {};
    a.r[0] = {dgu, 2 * (int64_t)fp};
    a.r[1] = {dgu + fp, 2 * (int64_t)fp};
    a.c[0] = {(const uint16_t*)wg, d.ld_w};
    a.c[1] = {(const uint16_t*)wu, d.ld_w};
    a.rows = d.m;
    a.cols = d.k;
    a.k = d.f;
    a.segments = 2;
    a.halves = 1;
    a.out[0] = gx;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && aligned_rows(a.c[1]) && d.k % 8 == 0;
    rc = run_gemm<false, true, OUT_PLAIN>(d.dtype, a, aligned, s);
  }
  if (rc == QCONV_OK && gwg) {
    GemmArgs a = {};
    a.r[0] = {dgu, 2 * (int64_t)fp};
    a.r[1] = {dgu + fp, 2 * (int64_t)fp};
    a.c[0] = {(const uint16_t*)x, d.ld_x};
    a.rows = d.f;
    a.cols = d.k;
    a.k = d.m;
    a.segments = 1;
    a.halves = 2;
    a.out[0] = gwg;
    a.out[1] = gwu;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && d.k % 8 == 0;
    rc = run_gemm<true, true, OUT_PLAIN>(d.dtype, a, aligned, s);
  }
  return rc;
}

}  // namespace qc
