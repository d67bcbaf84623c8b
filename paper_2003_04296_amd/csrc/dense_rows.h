// dense_rows.h -- products of a few tokens with a large weight matrix,
//   y[m][n] = sum_k x[m][k] w[n][k]  (plain with bias, or gated from two w),
// for 16-bit weights and for 4-bit ones with group scales.
//
// Bound by reading the weights once.  A block owns 16 outputs (16 rows of w)
// and 16 MT tokens; its waves take every NW-th block of 128 inputs, so all of
// w is in flight at once from many waves, and they are joined through LDS at
// the end.  Each load of a row is 16 bytes per lane.  The matrix instruction
// does the sums even for one token: its work is far below its rate, and it
// spares the reduction over lanes.  In its result a lane holds output
// lane % 16 and tokens (lane / 16) * 4 + 0..3, so one scale per lane and
// group serves 4-bit weights.
#pragma once

#include "dense.h"

namespace qc {

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

// What a wave reads of one block of 128 inputs.
template <class W, int H, int MT>
struct RowsBlock {
  static constexpr int SCALES = W::GROUP ? 128 / W::GROUP : 1;
  v4u x[MT][4];
  v4u w[H][W::GROUP ? 1 : 4];
  uint16_t s[H][SCALES];

  // FULL: all 128 inputs exist.  Otherwise what lies past k, or past the
  // codes and scales of the row, is zero and not read.
  template <bool FULL>
  __device__ __forceinline__ void load(const RowsArgs& a, const uint16_t* const xr[MT], const bool in[MT], int64_t row,
                                       int k0, int o) {
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
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = k0 + W::k_of(i, o);
        x[t][i] = v4u{0, 0, 0, 0};
        if (in[t]) x[t][i] = FULL ? load8(xr[t] + k) : load8_first(xr[t] + k, a.k - k);
      }
  }

  template <class T>
  __device__ __forceinline__ void multiply(v4f acc[H][MT]) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if constexpr (W::GROUP != 0) {
        uint32_t d[4] = {w[h][0][0], w[h][0][1], w[h][0][2], w[h][0][3]};
        W::arrange(d);
        v4u wf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          wf[i] = v4u{T::template from_e2m1<0>(d[i]), T::template from_e2m1<1>(d[i]), T::template from_e2m1<2>(d[i]),
                      T::template from_e2m1<3>(d[i])};
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int g = 0; g < SCALES; ++g) {
            v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = g * (4 / SCALES); i < (g + 1) * (4 / SCALES); ++i) sum = T::mfma(x[t][i], wf[i], sum);
            const float f = BF16::up(s[h][g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][t][e] = fmaf(f, sum[e], acc[h][t][e]);
          }
      } else {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[h][t] = T::mfma(x[t][i], w[h][i], acc[h][t]);
      }
    }
  }
};

// H = 1: y = sum + bias.  H = 2: y = act(sum 0) * sum 1.
template <class T, class W, int H, int MT, int NW, int U>
__global__ __launch_bounds__(NW * 64) void dense_rows_kernel(RowsArgs a) {
  __shared__ float part[NW][H][MT * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, o = lane >> 4;
  // workgroups go to the 8 dies in turn: the token tiles of one set of outputs
  // follow each other on one die, whose L2 then holds their weights
  const int nt = blockIdx.x / (8 * a.tiles_m) * 8 + blockIdx.x % 8, mt = blockIdx.x / 8 % a.tiles_m;
  if (nt >= a.tiles_n) return;
  const int n0 = nt * 16, m0 = mt * 16 * MT;
  const uint16_t* xr[MT];
  bool in[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    in[t] = m0 + t * 16 + r < a.m;
    xr[t] = a.x + (in[t] ? (int64_t)(m0 + t * 16 + r) * a.ld_x : 0);
  }
  const int64_t row = n0 + r < a.n ? n0 + r : 0;
  v4f acc[H][MT];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[h][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  const int full = a.k / 128, blocks = (a.k + 127) / 128;
  RowsBlock<W, H, MT> b[U];
  int kb = wave;
  for (; kb + (U - 1) * NW < full; kb += U * NW) {
#pragma unroll
    for (int u = 0; u < U; ++u) b[u].template load<true>(a, xr, in, row, (kb + u * NW) * 128, o);
#pragma unroll
    for (int u = 0; u < U; ++u) b[u].template multiply<T>(acc);
  }
  for (; kb < full; kb += NW) {
    b[0].template load<true>(a, xr, in, row, kb * 128, o);
    b[0].template multiply<T>(acc);
  }
  if (kb < blocks) {
    b[0].template load<false>(a, xr, in, row, kb * 128, o);
    b[0].template multiply<T>(acc);
  }
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][h][t * 256 + (o * 4 + e) * 16 + r] = acc[h][t][e];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += NW * 64) {
    const int m = m0 + i / 16, n = n0 + i % 16;
    if (m >= a.m || n >= a.n) continue;
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
}

// Tokens per block: 16 while the blocks do not fill the 256 compute units
// (weights read again come from L2), up to 64 otherwise, so that x is not read
// again for every 16 outputs.
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
    dense_rows_kernel<T, W, H, 4, NW, 1><<<(unsigned)blocks, NW * 64, 0, s>>>(a);
  else if (mt == 2)
    dense_rows_kernel<T, W, H, 2, NW, 1><<<(unsigned)blocks, NW * 64, 0, s>>>(a);
  else
    dense_rows_kernel<T, W, H, 1, NW, 2><<<(unsigned)blocks, NW * 64, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? QCONV_OK : QCONV_EHIP;
}

}  // namespace qc
