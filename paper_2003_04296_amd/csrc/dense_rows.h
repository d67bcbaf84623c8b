// dense_rows.h -- products of a few tokens with a large weight matrix,
//   y[m][n] = sum_k x[m][k] w[n][k]  (plain with bias, or gated from two w),
// for 16-bit weights and for 4-bit ones with group scales.
//
// Bound by reading the weights once, and past 16 tokens by x, which every
// block reads whole.  A block owns 16 outputs (16 rows of w) and its tokens;
// its waves take every NW-th block of 128 inputs, so all of w is in flight at
// once from many waves, and they are joined through LDS at the end.  Each load
// of a row is 16 bytes per lane.  The matrix instruction does the sums even for
// one token: its work is far below its rate, and it spares the reduction over
// lanes.  In its result a lane holds output lane % 16 and tokens
// (lane / 16) * 4 + 0..3, so one scale per lane and group serves 4-bit weights.
// Measured at 4096 x 4096 in 4 bits (8.9 MB), one call after the other in a
// graph, weights from the cache and from memory: one token 4.3 and 6.3 us (2.1
// and 1.4 TB/s; a kernel that reads the codes alone takes 3.3 from the cache), 16
// tokens 6.8 and 8.6, 32 10.4 and 11.7, 64 11.9 and 16.4.
#pragma once

#include "dense.h"
#include "qconv_internal.h"

namespace qc {

// The most tokens that take this way; from the next on, products go through
// tiles (dense_gemm.h).  us here and there in 4 bits, weights in the 256 MB cache:
//   4096 -> 4096   13.7 and 20.6 at 64 tokens, 20.3 and 22.0 at 80
//   4096 -> 16384  38.7 and 37.6, 70.1 and 38.1
//   2048 -> 8192   13.7 and 16.5, 21.2 and 17.4
//   8192 -> 1024   12.5 and 18.5, 17.2 and 18.9
// In 16 bits (gated, weights of 300 MB in turn) the two meet earlier: 22.3 and
// 24.2, 58 and 65, 18.0 and 23.4, 22.5 and 20.4 at 32 tokens, 28.2 and 25.6, 74
// and 68, 23.0 and 24.8, 22.8 and 21.2 at 64.
constexpr int ROWS_MOST = 64;

struct RowsArgs {
  const uint16_t* x;
  int64_t ld_x, ld_w, ld_y;
  const void* w[2];        // 16-bit values, or codes
  const uint16_t* sc[2];   // 4-bit weights: scales
  const float* bias;
  uint16_t* y;
  float* pre;              // gated: [m][2][ld_pre] or NULL
  int m, n, k, kp, act;    // kp: codes per row
  int ld_pre;
  int tiles_n, tiles_m;
};

// Swaps the upper 32 lanes of a with the lower 32 of b.
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
// Swaps rows 1 and 3 (of 16 lanes) of a with rows 0 and 2 of b.
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// 16-bit weights: in a block of 128 inputs, the i-th matrix instruction takes
// inputs [i * 32 + o * 8, +8) from lane row o.
struct Dense16 {
  static constexpr int GROUP = 0;
  __device__ __forceinline__ static int k_of(int i, int o) { return i * 32 + o * 8; }
};

// 4-bit weights.  Lane row o loads the 32 codes [o * 32, +32) of a row's 128
// in one 16-byte load; eight codes are one matrix operand.  An instruction may
// only mix inputs of one scale: with groups of 128 any will do, with 64 one
// exchange between the wave's halves puts each group into two instructions,
// with 32 two exchanges transpose the 4 x 4 pieces.
template <int G>
struct Q4 {
  static constexpr int GROUP = G;
  __device__ __forceinline__ static int k_of(int i, int o) {
    if constexpr (G == 128) return o * 32 + i * 8;
    if constexpr (G == 64) return (i >> 1) * 64 + (o & 1) * 32 + ((i & 1) + 2 * (o >> 1)) * 8;
    return i * 32 + o * 8;
  }
  __device__ __forceinline__ static void arrange(uint32_t d[4]) {
    if constexpr (G < 128) {
      swap32(d[0], d[2]);
      swap32(d[1], d[3]);
    }
    if constexpr (G == 64) {  // d = {0: A i0, 1: A i1, 2: B i0, 3: B i1}: k_of's order already
    }
    if constexpr (G == 32) {
      swap16(d[0], d[1]);
      swap16(d[2], d[3]);
    }
  }
};

// Whether all inputs [k0, k0 + 128) of k exist.  k0 may lie past k, where a
// pass is longer than what is left, and k0 + 128 past an int.
__host__ __device__ constexpr bool whole_block(int k, int k0) { return k - k0 >= 128; }
static_assert(whole_block(128, 0) && !whole_block(128, 1) && !whole_block(0x7fffff00, 0x7fffff80), "no overflow");

// A wave's weights in one block of 128 inputs.
template <class W, int H>
struct RowsBlock {
  static constexpr int SCALES = W::GROUP ? 128 / W::GROUP : 1;
  v4u w[H][W::GROUP ? 1 : 4];
  uint16_t s[H][SCALES];

  // FULL: all 128 inputs exist.  Otherwise what lies past k, or past the
  // codes and scales of the row, is zero and not read.
  template <bool FULL>
  __device__ __forceinline__ void load(const RowsArgs& a, int64_t row, int k0, int o) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if constexpr (W::GROUP != 0) {
        const bool on = FULL || k0 + o * 32 < a.kp;
        w[h][0] = on ? *(const v4u*)((const char*)a.w[h] + row * (a.kp / 2) + (k0 + o * 32) / 2) : v4u{0, 0, 0, 0};
        const uint16_t* sp = a.sc[h] + row * (a.kp / W::GROUP) + k0 / W::GROUP;
        if constexpr (FULL && SCALES == 4) {
          struct __attribute__((packed, aligned(2))) U {
            v2u v;
          };
          const v2u v = reinterpret_cast<const U*>(sp)->v;
          s[h][0] = (uint16_t)v[0], s[h][1] = (uint16_t)(v[0] >> 16);
          s[h][2] = (uint16_t)v[1], s[h][3] = (uint16_t)(v[1] >> 16);
        } else {
#pragma unroll
          for (int g = 0; g < SCALES; ++g) s[h][g] = FULL || k0 + g * W::GROUP < a.kp ? sp[g] : (uint16_t)0;
        }
      } else {
        const uint16_t* wr = (const uint16_t*)a.w[h] + row * a.ld_w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = k0 + W::k_of(i, o);
          w[h][i] = FULL ? load8(wr + k) : load8_first(wr + k, a.k - k);
        }
      }
    }
  }

  // x: the lane's token in LDS, at the block's first input; tiles of 16 tokens
  // `tile` values apart.
  template <class T, int MT>
  __device__ __forceinline__ void multiply(v4f (&acc)[H][MT], const uint16_t* x, int tile, int o) const {
    v4u wf[H][4];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if constexpr (W::GROUP != 0) {
        uint32_t d[4] = {w[h][0][0], w[h][0][1], w[h][0][2], w[h][0][3]};
        W::arrange(d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          wf[h][i] = v4u{T::template from_e2m1<0>(d[i]), T::template from_e2m1<1>(d[i]), T::template from_e2m1<2>(d[i]),
                         T::template from_e2m1<3>(d[i])};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) wf[h][i] = w[h][i];
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      v4u xf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xf[i] = *(const v4u*)(x + t * tile + W::k_of(i, o));
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (W::GROUP != 0) {
#pragma unroll
          for (int g = 0; g < SCALES; ++g) {
            v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = g * (4 / SCALES); i < (g + 1) * (4 / SCALES); ++i) sum = T::mfma(xf[i], wf[h][i], sum);
            const float f = BF16::up(s[h][g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][t][e] = fmaf(f, sum[e], acc[h][t][e]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[h][t] = T::mfma(xf[i], wf[h][i], acc[h][t]);
        }
      }
    }
  }
};

// H = 1: y = sum + bias.  H = 2: y = act(sum 0) * sum 1.
// A pass is NW blocks of 128 inputs, one per wave.  Its x lies in LDS, put
// there by all waves in whole rows; the next pass's x and weights are on their
// way into registers while it is multiplied.
template <class T, class W, int H, int MT, int NW>
__global__ __launch_bounds__(NW * 64) void dense_rows_kernel(RowsArgs a) {
  constexpr int PASS = NW * 128, LD = PASS + 8, WPT = PASS / 512, STEP = NW / WPT, PER = 16 * MT / STEP;
  __shared__ v4u xs[16 * MT * LD / 8];  // at the end: the waves' sums
  static_assert(sizeof(xs) >= sizeof(float) * NW * H * MT * 256, "sums fit");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, o = lane >> 4;
  // workgroups go to the 8 dies in turn: the token tiles of one set of outputs
  // follow each other on one die, whose L2 then holds their weights
  const int nt = blockIdx.x / (8 * a.tiles_m) * 8 + blockIdx.x % 8, mt = blockIdx.x / 8 % a.tiles_m;
  if (nt >= a.tiles_n) return;
  const int n0 = nt * 16, m0 = mt * 16 * MT;
  const int64_t row = n0 + r < a.n ? n0 + r : 0;
  v4f acc[H][MT];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[h][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  RowsBlock<W, H> b;
  v4u xr[PER];
  // A wave copies 512 inputs of every STEP-th token.  In place of those past
  // the last it takes that one; their results go nowhere.
  const int first = wave / WPT, col = (wave % WPT) * 512 + lane * 8;
  auto load = [&](int base) {
    const int k0 = base + wave * 128;
    if (whole_block(a.k, k0)) b.template load<true>(a, row, k0, o);
    else if (k0 < a.k) b.template load<false>(a, row, k0, o);
    const bool whole = a.k - base >= PASS;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int m = m0 + first + j * STEP, k = base + col;
      const uint16_t* p = a.x + (int64_t)(m < a.m ? m : a.m - 1) * a.ld_x + k;
      xr[j] = whole ? load8(p) : load8_first(p, a.k - k);
    }
  };
  load(0);
  for (uint32_t base = 0; base < (uint32_t)a.k; base += PASS) {
    if (base > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j) xs[(first + j * STEP) * (LD / 8) + col / 8] = xr[j];
    __syncthreads();
    const RowsBlock<W, H> now = b;
    if ((uint32_t)a.k - base > PASS) load(base + PASS);
    if ((int)base + wave * 128 < a.k)
      now.template multiply<T, MT>(acc, (const uint16_t*)xs + r * LD + wave * 128, 16 * LD, o);
  }
  __syncthreads();
  float* part = (float*)xs;  // [NW][H][MT * 256]
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[(wave * H + h) * (MT * 256) + t * 256 + (o * 4 + e) * 16 + r] = acc[h][t][e];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += NW * 64) {
    const int m = m0 + i / 16, n = n0 + i % 16;
    if (m >= a.m || n >= a.n) continue;
    float v[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      v[h] = part[h * (MT * 256) + i];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[h] += part[(w * H + h) * (MT * 256) + i];
    }
    float y;
    if constexpr (H == 2) {
      y = act_value(a.act, v[0]) * v[1];
      if (a.pre) {
        a.pre[(int64_t)m * 2 * a.ld_pre + n] = v[0];
        a.pre[((int64_t)m * 2 + 1) * a.ld_pre + n] = v[1];
      }
    } else {
      y = a.bias ? v[0] + a.bias[n] : v[0];
    }
    a.y[(int64_t)m * a.ld_y + n] = T::down(y);
  }
}

// The end of the kernels for at most 4 tokens: thread i < M * 16 joins the
// waves' sums of token i / 16 and output n0 + i % 16.
template <class T, int H, int M, int NW>
__device__ __forceinline__ void finish_few(const RowsArgs& a, const float (&part)[NW][H][M * 16], int n0) {
  __syncthreads();
  const int i = threadIdx.x, m = i / 16, n = n0 + i % 16;
  if (i >= M * 16 || m >= a.m || n >= a.n) return;
  float v[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    v[h] = part[0][h][i];
#pragma unroll
    for (int w = 1; w < NW; ++w) v[h] += part[w][h][i];
  }
  float y;
  if constexpr (H == 2) {
    y = act_value(a.act, v[0]) * v[1];
    if (a.pre) {
      a.pre[(int64_t)m * 2 * a.ld_pre + n] = v[0];
      a.pre[((int64_t)m * 2 + 1) * a.ld_pre + n] = v[1];
    }
  } else {
    y = a.bias ? v[0] + a.bias[n] : v[0];
  }
  a.y[(int64_t)m * a.ld_y + n] = T::down(y);
}

constexpr int FEW_MOST = 4;  // tokens they take

// At most 4 tokens on 4-bit weights.  Lane row o holds 32 codes of one group,
// and the row of x's operand that stands for token t and lane row o is zero in
// the other lane rows: the matrix instruction's 16 rows, of which tokens would
// fill 4 at most, keep the lane rows' sums apart.  So the codes need no
// exchange between lanes, whatever the group, a lane needs one scale per 32
// codes instead of up to four, and the scales take one fma per token.
// x lies in LDS, PASS inputs at a time, and lanes that stand for no token read
// zeros there: no load is conditional (a branch around them made the compiler
// copy all operands).  Gated 4096 -> 16384 in groups of 32, in us from the cache:
// 17.6 for one token and 21.5 for four, against 20.6 and 23 of a form like
// dense_rows_kernel's; reading the codes alone takes 10.7.  From memory 19.0 and
// 23.9.
template <class T, int GROUP, int H, int M, int NW>
__global__ __launch_bounds__(NW * 64) void dense_few_kernel(RowsArgs a) {
  constexpr int PASS = 4096, LD = PASS + 8;  // + 8: the tokens' values in different banks
  static_assert(PASS % (NW * 128) == 0, "a pass is whole rounds");
  __shared__ float part[NW][H][M * 16];
  __shared__ v4u xs[(M * LD + 128) / 8];  // the tokens, then zeros
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, o = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const bool in = r >> 2 == o && (r & 3) < M;
  const int64_t row = n0 + r < a.n ? n0 + r : 0;
  const char* wr[H];
  const uint16_t* sr[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    wr[h] = (const char*)a.w[h] + row * (a.kp / 2);
    sr[h] = a.sc[h] + row * (a.kp / GROUP);
  }
  float acc[H][M];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < M; ++t) acc[h][t] = 0.0f;
  v4u w[H];
  float sc[H];
  // 32 codes of input k0 + o * 32; past the row its last ones, with a scale of
  // zero (x is zero there, too, but a scale may be an infinity)
  auto load = [&](int k0) {
    const int k = k0 + o * 32, c = k < a.kp ? k : a.kp - 32;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      w[h] = *(const v4u*)(wr[h] + (uint32_t)c / 2);
      sc[h] = k < a.kp ? BF16::up(sr[h][(uint32_t)c / GROUP]) : 0.0f;
    }
  };
  if (threadIdx.x < 16) xs[M * LD / 8 + threadIdx.x] = v4u{0, 0, 0, 0};
  for (uint32_t base = 0; base < (uint32_t)a.k; base += PASS) {
    const int here = a.k - base < PASS ? a.k - base : PASS, blocks = (here + 127) / 128;
    if (wave < blocks) load(base + wave * 128);
    if (base > 0) __syncthreads();
#pragma unroll
    for (int t = 0; t < M; ++t)
      for (int i = threadIdx.x; i < blocks * 16; i += NW * 64)
        xs[t * (LD / 8) + i] = t < a.m ? load8_first(a.x + t * a.ld_x + base + i * 8, here - i * 8) : v4u{0, 0, 0, 0};
    __syncthreads();
    const char* xp = (const char*)xs + (in ? ((r & 3) * LD + wave * 128 + o * 32) * 2 : M * LD * 2);
    const int by = in ? NW * 256 : 0;
    for (int kb = wave; kb < blocks; kb += NW) {
      v4u x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *(const v4u*)(xp + i * 16);
      xp += by;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
        const v4u c = w[h];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum = T::mfma(x[i], v4u{T::template from_e2m1<0>(c[i]), T::template from_e2m1<1>(c[i]),
                                  T::template from_e2m1<2>(c[i]), T::template from_e2m1<3>(c[i])}, sum);
#pragma unroll
        for (int t = 0; t < M; ++t) acc[h][t] = fmaf(sc[h], sum[t], acc[h][t]);
      }
      if (kb + NW < blocks) load(base + (kb + NW) * 128);
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < M; ++t) {
      float v = acc[h][t];
      v += __shfl_xor(v, 16);
      v += __shfl_xor(v, 32);
      if (o == 0) part[wave][h][t * 16 + r] = v;
    }
  finish_few<T, H, M, NW>(a, part, n0);
}

// At most 4 tokens on 16-bit weights: two blocks of 128 inputs are under way
// per wave.  Lanes past the tokens keep zeros.  No LDS for x: what is waited for
// is the weights, and a barrier before the first product costs more (2048 ->
// 8192, one token, two weights: 12.3 us against 11.7).
template <class T, int H, int NW>
__global__ __launch_bounds__(NW * 64) void dense_few16_kernel(RowsArgs a) {
  constexpr int M = FEW_MOST, U = 2;
  __shared__ float part[NW][H][M * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, o = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const bool in = r < a.m;
  const uint16_t* xr = a.x + (in ? (int64_t)r * a.ld_x : 0) + o * 8;
  const uint16_t* wr[H];
#pragma unroll
  for (int h = 0; h < H; ++h) wr[h] = (const uint16_t*)a.w[h] + (int64_t)(n0 + r < a.n ? n0 + r : 0) * a.ld_w + o * 8;
  v4f acc[H];
#pragma unroll
  for (int h = 0; h < H; ++h) acc[h] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  v4u x[U][4] = {}, w[U][H][4];
  auto load = [&](int u, int k0) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[u][h][i] = load8(wr[h] + k0 + i * 32);
    if (in) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[u][i] = load8(xr + k0 + i * 32);
    }
  };
  auto multiply = [&](int u) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[h] = T::mfma(x[u][i], w[u][h][i], acc[h]);
  };
  const int full = a.k / 128;
  int kb = wave;
  for (; kb + (U - 1) * NW < full; kb += U * NW) {
#pragma unroll
    for (int u = 0; u < U; ++u) load(u, (kb + u * NW) * 128);
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(u);
  }
  for (; kb < full; kb += NW) {
    load(0, kb * 128);
    multiply(0);
  }
  if (kb < (a.k + 127) / 128) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = kb * 128 + i * 32, left = a.k - k - o * 8;
      x[0][i] = load8_first(xr + k, in ? left : 0);
#pragma unroll
      for (int h = 0; h < H; ++h) w[0][h][i] = load8_first(wr[h] + k, left);
    }
    multiply(0);
  }
  if (o == 0) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int t = 0; t < M; ++t) part[wave][h][t * 16 + r] = acc[h][t];
  }
  finish_few<T, H, M, NW>(a, part, n0);
}

// GROUP 0: 16-bit weights.
template <class T, int GROUP, int H>
int run_dense_few(RowsArgs& a, hipStream_t s) {
  constexpr int NW = 8;
  const int blocks = ceil_div(a.n, 16);
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  if constexpr (GROUP == 0)
    dense_few16_kernel<T, H, NW><<<blocks, NW * 64, 0, s>>>(a);
  else if (a.m == 1)
    dense_few_kernel<T, GROUP, H, 1, NW><<<blocks, NW * 64, 0, s>>>(a);
  else
    dense_few_kernel<T, GROUP, H, FEW_MOST, NW><<<blocks, NW * 64, 0, s>>>(a);
  return hip_status();
}

// Tokens per block: 16 while the blocks do not fill the 256 compute units
// (weights read again come from L2), up to 64 otherwise, so that x is not read
// again for every 16 outputs.  From 32 on four waves per block, whose x leaves
// LDS for two or more blocks per unit: 4-bit 4096 -> 16384 for 64 tokens 39 us
// against 56 with eight, gated for 32 tokens 36 against 43.  A single block per
// unit and long rows: sixteen, half as many passes one after the other (4-bit
// 8192 -> 1024 for 64 tokens, weights not in the caches: 14.4 us against 16.8).
template <class T, class W, int H>
int run_dense_rows(RowsArgs& a, hipStream_t s) {
  constexpr int NW = 8;
  a.tiles_n = (a.n + 15) / 16;
  const int mts = (a.m + 15) / 16;
  const int64_t enough = 512;
  const int mt = mts >= 4 && (int64_t)a.tiles_n * ((mts + 3) / 4) >= enough ? 4
                 : mts >= 2 && (int64_t)a.tiles_n * ((mts + 1) / 2) >= enough ? 2 : 1;
  a.tiles_m = (mts + mt - 1) / mt;
  const int64_t blocks = (int64_t)(a.tiles_n + 7) / 8 * 8 * a.tiles_m;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  if (mt == 4)
    dense_rows_kernel<T, W, H, 4, 4><<<(unsigned)blocks, 4 * 64, 0, s>>>(a);
  else if (mt == 2)
    dense_rows_kernel<T, W, H, 2, 4><<<(unsigned)blocks, 4 * 64, 0, s>>>(a);
  else if (blocks <= 256 && a.k > NW * 128)
    dense_rows_kernel<T, W, H, 1, 2 * NW><<<(unsigned)blocks, 2 * NW * 64, 0, s>>>(a);
  else
    dense_rows_kernel<T, W, H, 1, NW><<<(unsigned)blocks, NW * 64, 0, s>>>(a);
  return hip_status();
}

}  // namespace qc
