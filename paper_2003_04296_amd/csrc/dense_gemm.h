// dense_gemm.h -- C[r][c] = sum_k R(r, k) Q(c, k) on the matrix cores for many
// rows: the three products of the feed-forward block in 16-bit types, and
// those with 4-bit weights for more tokens than dense_rows.h takes.
//
// Operands whose k runs along their rows ("row form": x, W in the forward,
// dg/du in gx) are read from LDS as 16 bytes per lane, operands whose k runs
// down their columns ("column form": W in gx, all of gW) through the
// transposing LDS reads.  4-bit weights are expanded on their way into LDS.
#pragma once

#include <type_traits>

#include "dense.h"
#include "qconv_internal.h"

namespace qc {

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
  // 4-bit weights in place of c: codes, scales, and a power of two per row
  // that keeps scale * magnitude inside fp16 (NULL for bf16)
  const uint8_t* codes[2];
  const uint16_t* scales[2];
  const float* unit[2];
  int kp;  // codes per row
  void* out[2];
  int64_t ld_out;
  int wide_out;  // rows of out start at 8-byte addresses
  const float* bias;
  float* pre;  // OUT_GATED: [rows][2][ld_pre] or NULL
  int ld_pre;
  int act;
  // the products of a tile split over `parts` blocks: fp32 sums go to
  // part[parts][2 or halves][rows][ld_part], joined by dense_join_kernel
  int parts;
  float* part;
  int ld_part;
};

// LDS holds chunks of 16 bytes.  Row form: rows of 64 products (8 chunks)
// with the chunk index xored by the row, so that the 16 rows of a fragment
// read lie in different banks.  Column form: one LDS row per product, of ROWS
// values; a transposing read touches 4 of them at one place, and the lanes
// beside it 4 more 8 rows below, which the xor spreads over the banks.
__device__ __forceinline__ int swz_row(int r) { return r & 7; }
__device__ __forceinline__ int swz_col(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) << 1; }

// Columns of the gated forward: 64 columns of the tile are 32 gate rows and
// the 32 up rows of the same hidden features, so that one lane ends up with
// both sums.  The weight row of tile column t.
template <bool PAIR>
__device__ __forceinline__ int weight_row(int t) {
  return PAIR ? (t / 64) * 32 + t % 32 : t;
}

// The tile of one 16-bit operand: ROWS rows (or columns) of C by KSTEP
// products, staged by NT threads, CH chunks each.  SIDE 0: GemmArgs::r, 1: c.
//
// ALIGNED: every row of the operand starts at a 16-byte address and the rows'
// length (k in row form) is a multiple of 8, so each chunk is one 16-byte load
// straight into LDS; chunks past the ends get an offset past the buffer's
// range, which loads zeros.  Otherwise chunks pass through registers, and the
// ones that cross an end are read value by value.
template <int ROWS, int NT, int SIDE, bool COL_, bool ALIGNED, bool PAIR>
struct Stage16 {
  static constexpr bool COL = COL_, DIRECT = ALIGNED;
  static constexpr int CH = ROWS * KSTEP / 8 / NT;
  const uint16_t *p, *p2;  // the tile's first value, product 0
  int64_t ld;
  int rows;  // rows of the operand from the tile's first (gate rows for PAIR)
  typedef std::conditional_t<ALIGNED, uint32_t, int64_t> Off;
  static constexpr Off OUTSIDE = ALIGNED ? (Off)0x80000000u : (Off)-1;
  Off off[CH];  // byte offset of each chunk from p, or OUTSIDE
  int at[CH];   // its first product (row form) or its product (column form)
  v4u reg[ALIGNED ? 1 : CH];

  __device__ __forceinline__ static int chunk(int j) { return (int)threadIdx.x + j * NT; }

  __device__ __forceinline__ void init(const GemmArgs& a, int which, int64_t r0) {
    const Operand& o = SIDE == 0 ? a.r[which] : a.c[which];
    const int64_t all = SIDE == 0 ? a.rows : a.cols;
    p = o.p + (COL ? r0 : r0 * o.ld);
    p2 = PAIR ? a.c[1].p + r0 * o.ld : nullptr;
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
        const int r = weight_row<PAIR>(t);
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

// The tile of 4-bit weights, in row form: a thread takes 32 codes of one row
// (of one group) and writes them to LDS as scale * magnitude in the 16-bit
// type.  That is exact: the scales have 6 significant bits, the magnitudes 2.
// In fp16 a row's scales are first divided by a power of two near the largest
// of them, multiplied back into the sums; only groups whose scale is more than
// 2^18 below the row's largest are rounded then, to 2^-25 of that one.
template <class T, int ROWS, int NT, int GROUP, bool PAIR>
struct StageQ4 {
  static constexpr bool COL = false, DIRECT = false;
  static_assert(ROWS * KSTEP / 32 == NT, "one piece per thread");
  const uint8_t* p;
  const uint16_t* sp;
  float unit;
  int kp;
  bool in;
  v4u code;
  uint16_t sc;

  __device__ __forceinline__ void init(const GemmArgs& a, int, int64_t r0) {
    const int t = threadIdx.x / 2, half = PAIR && (t & 32) ? 1 : 0;
    const int64_t row = r0 + weight_row<PAIR>(t);
    in = row < a.cols;
    kp = a.kp;
    p = a.codes[half] + (in ? row : 0) * (kp / 2);
    sp = a.scales[half] + (in ? row : 0) * (kp / GROUP);
    unit = a.unit[half] && in ? a.unit[half][row] : 1.0f;
  }
  __device__ __forceinline__ void load(v4u*, int k0, int) {
    const int k = k0 + (threadIdx.x & 1) * 32;
    const bool on = in && k < kp;
    code = on ? *(const v4u*)(p + k / 2) : v4u{0, 0, 0, 0};
    sc = on ? sp[k / GROUP] : (uint16_t)0;
  }
  __device__ __forceinline__ void store(v4u* lds) {
    const int t = threadIdx.x / 2, h = threadIdx.x & 1;
    const float s = BF16::up(sc) * unit;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t c = code[q];
      lds[t * 8 + ((h * 4 + q) ^ swz_row(t))] = v4u{T::template scaled_e2m1<0>(c, s), T::template scaled_e2m1<1>(c, s),
                                                    T::template scaled_e2m1<2>(c, s), T::template scaled_e2m1<3>(c, s)};
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

// The order of a stage's LDS reads and matrix instructions.  Left alone, the
// compiler reads each fragment right before its use, and the wave waits out
// the LDS latency a dozen times per stage.  Here the first fragments are read
// ahead and the rest are spread evenly over the first two thirds of the
// instructions, a few fragments before their use: FC and FR reads make one
// fragment of a column group (4 in a half stage) and of a row group (NR).
template <int NR, int FC, int FR>
struct ReadOrder {
  static constexpr int ALL = 2 * (4 * FC + NR * FR), FIRST = 4 * FC + 3 * FR, GROUPS = 2 * NR;
  static constexpr int before(int g) {  // reads issued before group g of 4 instructions
    const int n = FIRST + ((ALL - FIRST) * g * 3 + 2 * GROUPS - 1) / (2 * GROUPS);
    return n < ALL ? n : ALL;
  }
};
template <int NR, int FC, int FR>
__device__ __forceinline__ void order_reads() {
  typedef ReadOrder<NR, FC, FR> O;
  constexpr int MFMA = 0x8, DS_READ = 0x100;
  __builtin_amdgcn_sched_group_barrier(DS_READ, O::FIRST, 0);
  Unroll<0, O::GROUPS>::run([](auto g) {
    constexpr int G = decltype(g)::value;
    __builtin_amdgcn_sched_group_barrier(MFMA, 4, 0);
    if constexpr (O::before(G + 1) > O::before(G))
      __builtin_amdgcn_sched_group_barrier(DS_READ, O::before(G + 1) - O::before(G), 0);
  });
}

// Results of row r, columns c..c + 3: bias, activation, rounding, store.
template <class T, int OUT>
__device__ __forceinline__ void finish4(const GemmArgs& a, int half, int64_t r, int64_t c, float v[2][4]) {
  if constexpr (OUT == OUT_GATED) {
    if (a.pre) {
      float* g = a.pre + r * 2 * a.ld_pre + c;
      if (c + 4 <= a.cols) {
        *(v4f*)g = v4f{v[0][0], v[0][1], v[0][2], v[0][3]};
        *(v4f*)(g + a.ld_pre) = v4f{v[1][0], v[1][1], v[1][2], v[1][3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.cols) {
            g[e] = v[0][e];
            g[a.ld_pre + e] = v[1][e];
          }
      }
    }
    float h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = act_value(a.act, v[0][e]) * v[1][e];
    put4<T>(a.out[0], r * a.ld_out, c, a.cols, a.wide_out, h);
  } else {
    if (a.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < a.cols) v[0][e] += a.bias[c + e];
    }
    put4<T>(a.out[half], r * a.ld_out, c, a.cols, a.wide_out, v[0]);
  }
}

// A block computes a BR x BC tile of C with waves of (BR / 2) x 64 each.
// Two LDS stages: while the waves multiply one, the next is loaded.
template <class T, class SR, class SC, int OUT, int BR, int BC>
__global__ __launch_bounds__(BC / 64 * 128) void dense_gemm_kernel(GemmArgs a) {
  constexpr int NR = BR / 32, PAIR = OUT == OUT_GATED;
  constexpr int LR = BR * KSTEP / 8, LC = BC * KSTEP / 8;
  __shared__ v4u lds[2][LR + LC];
  // Workgroups go to the 8 dies in turn; each die gets a run of tiles that
  // share operands in its L2: 8 tile rows at a time, column after column.
  const uint32_t trs = a.tiles_r * a.halves, all = trs * a.tiles_c, group = 8 * a.tiles_c;
  const uint32_t id = blockIdx.x % all, part = blockIdx.x / all, die = id & 7;
  const uint32_t tile = die * (all / 8) + (die < all % 8 ? die : all % 8) + id / 8;
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

  SR sr;
  SC sc;
  const int steps = ceil_div(a.k, KSTEP), total = steps * a.segments;
  const int begin = (int)((int64_t)total * part / a.parts), end = (int)((int64_t)total * (part + 1) / a.parts);
  int seg = begin >= steps, k0 = (begin - seg * steps) * KSTEP;
  sr.init(a, seg + half, r0);
  sc.init(a, seg, c0);
  if (begin < end) {
    sr.load(lds[0], k0, a.k);
    sc.load(lds[0] + LR, k0, a.k);
    sr.store(lds[0]);
    sc.store(lds[0] + LR);
  }
  for (int step = begin; step < end; ++step) {
    const int b = (step - begin) & 1;
    if constexpr (SR::DIRECT || SC::DIRECT)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads into LDS are not waited for elsewhere
    lds_barrier();
    k0 += KSTEP;
    if (step + 1 == steps && a.segments == 2) {
      sr.init(a, 1, r0);
      sc.init(a, 1, c0);
      k0 = 0;
    }
    if (step + 1 < end) {
      sr.load(lds[b ^ 1], k0, a.k);
      sc.load(lds[b ^ 1] + LR, k0, a.k);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      v4u fr[NR], fc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) fc[i] = fragment<BC, SC::COL>(lds[b] + LR, wc + i * 16, s);
#pragma unroll
      for (int i = 0; i < NR; ++i) fr[i] = fragment<BR, SR::COL>(lds[b], wr + i * 16, s);
#pragma unroll
      for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = T::mfma(fc[i], fr[j], acc[i][j]);
    }
    order_reads<NR, SC::COL ? 2 : 1, SR::COL ? 2 : 1>();
    if (step + 1 < end) {
      sr.store(lds[b ^ 1]);
      sc.store(lds[b ^ 1] + LR);
    }
  }
#pragma unroll
  for (int i = 0; i < (PAIR ? 2 : 4); ++i) {
    const int64_t c = c0 + (PAIR ? wc / 2 : wc) + i * 16 + (lane >> 4) * 4;
    float back[2][4];  // what the 4-bit weights' rows were divided by
#pragma unroll
    for (int h = 0; h < (PAIR ? 2 : 1); ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) back[h][e] = a.unit[h] && c + e < a.cols ? 1.0f / a.unit[h][c + e] : 1.0f;
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      const int64_t r = r0 + wr + j * 16 + (lane & 15);
      if (r >= a.rows || c >= a.cols) continue;
      float v[2][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[0][e] = acc[i][j][e] * back[0][e];
        if constexpr (PAIR) v[1][e] = acc[i + 2][j][e] * back[1][e];
      }
      if (a.parts > 1) {
#pragma unroll
        for (int h = 0; h < (PAIR ? 2 : 1); ++h)
          *(v4f*)(a.part + (((int64_t)part * (PAIR ? 2 : a.halves) + (PAIR ? h : half)) * a.rows + r) * a.ld_part + c) =
              v4f{v[h][0], v[h][1], v[h][2], v[h][3]};
        continue;
      }
      finish4<T, OUT>(a, half, r, c, v);
    }
  }
}

// Joins the parts of a split product: four columns of one row per thread.
template <class T, int OUT>
__global__ __launch_bounds__(256) void dense_join_kernel(GemmArgs a) {
  constexpr int H = OUT == OUT_GATED ? 2 : 1;
  const int q = a.ld_part / 4;
  const int64_t n = (int64_t)a.rows * q * (OUT == OUT_GATED ? 1 : a.halves);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / q;  // of both halves
    const int half = row >= a.rows;
    const int64_t c = i % q * 4;
    const int64_t plane = (int64_t)a.rows * a.ld_part, step = plane * (OUT == OUT_GATED ? 2 : a.halves);
    float v[2][4];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float* p = a.part + h * plane + row * a.ld_part + c;
      v4f s = *(const v4f*)p;
      for (int k = 1; k < a.parts; ++k) s += *(const v4f*)(p + k * step);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[h][e] = s[e];
    }
    finish4<T, OUT>(a, half, row - half * (int64_t)a.rows, c, v);
  }
}

// Every row of the operand starts at a 16-byte address, and a tile's offsets
// stay below 2^31 bytes.
inline bool aligned_rows(const Operand& o) {
  return ((uintptr_t)o.p & 15) == 0 && o.ld % 8 == 0 && o.ld < (1 << 21);
}

// How many blocks share a tile's products: enough that the chip is filled,
// while each keeps at least 8 steps.
inline int gemm_parts(int64_t tiles, int64_t steps) {
  if (tiles >= 192) return 1;
  int64_t p = 512 / tiles;
  if (p > steps / 8) p = steps / 8;
  return p < 1 ? 1 : (int)(p < 64 ? p : 64);
}

struct GemmPlan {
  int tile;  // rows and columns of a block's tile
  int parts;
  size_t bytes;  // of GemmArgs::part
};

// 256 x 256 tiles where they fill the chip by themselves; else 128 x 128, the
// products split where those do not either.  `out` = columns of C per tile
// column (a gated tile makes half as many).
inline GemmPlan gemm_plan(int64_t rows, int64_t cols, int64_t steps, int halves, bool gated, bool aligned) {
  auto tiles = [&](int b) { return (rows + b - 1) / b * ((cols + (gated ? b / 2 : b) - 1) / (gated ? b / 2 : b)) * halves; };
  if (aligned && tiles(256) >= 256) return {256, 1, 0};
  GemmPlan p = {128, gemm_parts(tiles(128) ? tiles(128) : 1, steps), 0};
  if (p.parts > 1) p.bytes = (size_t)p.parts * (gated ? 2 : halves) * rows * round_up(cols, 4) * 4;
  return p;
}

template <class T, class SR, class SC, int OUT, int B>
int run_gemm_tiles(GemmArgs& a, hipStream_t s) {
  a.tiles_r = ceil_div(a.rows, B);
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? B / 2 : B);
  const int64_t blocks = (int64_t)a.tiles_r * a.tiles_c * a.halves * a.parts;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  a.ld_part = (int)round_up(a.cols, 4);
  a.wide_out = a.ld_out % 4 == 0 && ((uintptr_t)a.out[0] & 7) == 0 && ((uintptr_t)a.out[1] & 7) == 0;
  dense_gemm_kernel<T, SR, SC, OUT, B, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a);
  if (a.parts > 1) {
    const int64_t n = (int64_t)a.rows * (a.ld_part / 4) * (OUT == OUT_GATED ? 1 : a.halves);
    dense_join_kernel<T, OUT><<<(unsigned)(n < (1 << 20) ? (n + 255) / 256 : 4096), 256, 0, s>>>(a);
  }
  return hip_status();
}

}  // namespace qc
