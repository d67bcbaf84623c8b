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
#include "dense.h"

#include "qconv_internal.h"

namespace qc {

namespace {

constexpr int TILE = 128;  // rows and columns of C per block
constexpr int KSTEP = 64;  // products per LDS stage

// One operand: `rows` of C's rows (or columns) and `k` products.  Row form:
// value (r, k) at p[r * ld + k]; column form: at p[k * ld + r].
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
  float* pre;  // OUT_GATED: [rows][2][ld_pre] or NULL
  int ld_pre;
  int act;
};

// Chunks of 16 bytes.  Row form: LDS rows of 64 products (8 chunks) with the
// chunk index xored by the row, so that the 16 rows a fragment read touches
// lie in different banks.  Column form: LDS rows of 128 C-rows (16 chunks);
// a transposing read touches 4 or 8 LDS rows at one place, which the xor
// spreads over all banks.
__device__ __forceinline__ int swz_col(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) << 1; }

template <bool COL>
__device__ __forceinline__ void load_tile(v4u* lds, const Operand& o, int64_t r0, int rows, int k0, int k) {
#pragma unroll
  for (int j = 0; j < TILE * KSTEP / 8 / 256; ++j) {
    const int p = threadIdx.x + j * 256;
    if constexpr (!COL) {
      const int r = p / 8, c = (p % 8) ^ (r & 7);
      const bool in = r0 + r < rows;
      lds[p] = load8_first(o.p + (in ? (r0 + r) * o.ld + k0 + c * 8 : 0), in ? k - (k0 + c * 8) : 0);
    } else {
      const int kk = p / 16, c = (p % 16) ^ swz_col(kk);
      const bool in = k0 + kk < k;
      lds[p] = load8_first(o.p + (in ? (int64_t)(k0 + kk) * o.ld + r0 + c * 8 : 0), in ? (int)(rows - (r0 + c * 8)) : 0);
    }
  }
}

// The gated forward's columns: 64 columns of the tile are 32 gate rows and
// the 32 up rows of the same hidden features, so that one lane ends up with
// both sums.
__device__ __forceinline__ void load_tile_gated(v4u* lds, const Operand& g, const Operand& u, int f0, int f, int k0,
                                                int k) {
#pragma unroll
  for (int j = 0; j < TILE * KSTEP / 8 / 256; ++j) {
    const int p = threadIdx.x + j * 256;
    const int r = p / 8, c = (p % 8) ^ (r & 7);
    const int row = f0 + (r / 64) * 32 + r % 32;
    const Operand& o = (r & 32) ? u : g;
    const bool in = row < f;
    lds[p] = load8_first(o.p + (in ? row * o.ld + k0 + c * 8 : 0), in ? k - (k0 + c * 8) : 0);
  }
}

// The 8 products [s * 32 + (lane / 16) * 8, +8) of tile row r0 + lane % 16.
template <bool COL>
__device__ __forceinline__ v4u fragment(const v4u* lds, int r0, int s) {
  const int lane = threadIdx.x & 63;
  if constexpr (!COL) {
    const int r = r0 + (lane & 15);
    return lds[r * 8 + ((s * 4 + (lane >> 4)) ^ (r & 7))];
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
      const char* at = (const char*)(lds + k * 16 + (c ^ swz_col(k))) + (lane & 1) * 8;
      h[j] = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)at));
    }
    return v4u{h[0][0], h[0][1], h[1][0], h[1][1]};
  }
}

template <class T, bool RCOL, bool CCOL, int OUT>
__global__ __launch_bounds__(256) void ffn_gemm_kernel(GemmArgs a) {
  __shared__ v4u lr[TILE * KSTEP / 8], lc[TILE * KSTEP / 8];
  const int tile = blockIdx.x % (a.tiles_r * a.tiles_c), half = blockIdx.x / (a.tiles_r * a.tiles_c);
  const int64_t r0 = (int64_t)(tile % a.tiles_r) * TILE;
  const int64_t c0 = (int64_t)(tile / a.tiles_r) * (OUT == OUT_GATED ? TILE / 2 : TILE);
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int wr = (wave & 1) * 64, wc = (wave >> 1) * 64;
  v4f acc[4][4];  // [column group][row group]: lane holds row lane % 16, columns (lane / 16) * 4 + 0..3
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int seg = 0; seg < a.segments; ++seg) {
    for (int k0 = 0; k0 < a.k; k0 += KSTEP) {
      __syncthreads();
      load_tile<RCOL>(lr, a.r[seg + half], r0, a.rows, k0, a.k);
      if constexpr (OUT == OUT_GATED)
        load_tile_gated(lc, a.c[0], a.c[1], (int)c0, a.cols, k0, a.k);
      else
        load_tile<CCOL>(lc, a.c[seg], c0, a.cols, k0, a.k);
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        v4u fr[4], fc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          fr[i] = fragment<RCOL>(lr, wr + i * 16, s);
          fc[i] = fragment<CCOL>(lc, wc + i * 16, s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(fc[i], fr[j], acc[i][j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = r0 + wr + j * 16 + (lane & 15);
    if (r >= a.rows) continue;
    if constexpr (OUT == OUT_GATED) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t f = c0 + wc / 2 + i * 16 + (lane >> 4) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (f + e >= a.cols) continue;
          const float g = acc[i][j][e], u = acc[i + 2][j][e];
          ((uint16_t*)a.out[0])[r * a.ld_out + f + e] = T::down(act_value(a.act, g) * u);
          if (a.pre) {
            a.pre[r * 2 * a.ld_pre + f + e] = g;
            a.pre[(r * 2 + 1) * a.ld_pre + f + e] = u;
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t c = c0 + wc + i * 16 + (lane >> 4) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.cols) ((uint16_t*)a.out[half])[r * a.ld_out + c + e] = T::down(acc[i][j][e]);
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

template <bool RCOL, bool CCOL, int OUT>
int run_gemm(int dtype, GemmArgs& a, hipStream_t s) {
  a.tiles_r = ceil_div(a.rows, TILE);
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? TILE / 2 : TILE);
  const int64_t blocks = (int64_t)a.tiles_r * a.tiles_c * a.halves;
  if (blocks >= (1 << 24)) return QCONV_EUNSUPPORTED;  // 2^32 threads
  if (dtype == QCONV_F16)
    ffn_gemm_kernel<F16, RCOL, CCOL, OUT><<<(unsigned)blocks, 256, 0, s>>>(a);
  else
    ffn_gemm_kernel<BF16, RCOL, CCOL, OUT><<<(unsigned)blocks, 256, 0, s>>>(a);
  return hip_status();
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
  return run_gemm<false, false, OUT_GATED>(d.dtype, a, s);
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
    rc = run_gemm<false, true, OUT_PLAIN>(d.dtype, a, s);
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
    rc = run_gemm<true, true, OUT_PLAIN>(d.dtype, a, s);
  }
  return rc;
}

}  // namespace qc
