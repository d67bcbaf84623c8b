// q4.hip -- weights of 4 bits with group scales: packing, and the products
//   y = x W^T + bias,   h = act(x Wg^T) * (x Wu^T)
// with W = scale * E2M1 magnitude, whatever bf16 value the scale is.  No weight is
// rounded: for few tokens the codes become 16-bit operands by the conversion
// instruction (exact), one matrix instruction sums 32 products of a group, and
// the group's fp32 sum is multiplied by its scale; for many the operands are
// scale * magnitude, and a tile with scales whose products 16 bits do not hold is
// summed in two parts or group by group (dense_gemm.h).
#include "dense_gemm.h"
#include "dense_rows.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// ---------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------

// fp32 bits rounded to 6 significant bits, to nearest, ties to even.
__device__ __forceinline__ uint32_t round6(uint32_t b) { return (b + 0x1FFFFu + ((b >> 18) & 1u)) & ~0x3FFFFu; }

// Nearest magnitude's index of r >= 0; a tie takes the smaller.
__device__ __forceinline__ uint32_t e2m1_index(float r) {
  return (r > 0.25f) + (r > 0.75f) + (r > 1.25f) + (r > 1.75f) + (r > 2.5f) + (r > 3.5f) + (r > 5.0f);
}

template <int DT>
__device__ __forceinline__ float load_value(const void* p, int64_t i) {
  if constexpr (DT == QCONV_F32) return ((const float*)p)[i];
  if constexpr (DT == QCONV_F16) return F16::up(((const uint16_t*)p)[i]);
  return BF16::up(((const uint16_t*)p)[i]);
}

// Eight values of a group per thread, group / 8 neighbouring lanes a group.
// Once per weight: 16384 x 16384 values take 460 us in fp32 and 380 in 16 bits (2.6
// and 1.8 TB/s), bound by the loads, one value each, that rows at any address allow.
template <int DT>
__global__ __launch_bounds__(256) void q4_pack_kernel(const void* __restrict__ w, int n, int k, int64_t ld, int group,
                                                      int kp, float top, uint32_t* __restrict__ codes,
                                                      uint16_t* __restrict__ scales) {
  const int per = group / 8;  // 4, 8 or 16 lanes
  const int64_t units = (int64_t)n * (kp / 8), padded = (units + 255) / 256 * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < padded; i += (int64_t)gridDim.x * 256) {
    const bool on = i < units;
    const int64_t row = on ? i / (kp / 8) : 0;
    const int c = on ? (int)(i % (kp / 8)) * 8 : kp;
    float v[8], big = 0.0f;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = c + e < k ? load_value<DT>(w, row * ld + c + e) : 0.0f;
      big = fmaxf(big, fabsf(v[e]));
      odd |= !(fabsf(v[e]) < __builtin_inff());
    }
    uint32_t bad = odd;
    for (int d = 1; d < per; d *= 2) {
      big = fmaxf(big, __shfl_xor(big, d));
      bad |= __shfl_xor(bad, d);
    }
    const float s = __uint_as_float(round6(__float_as_uint(big / top)));
    uint32_t code = 0;
    if (s > 0.0f && !bad) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t mag = e2m1_index(fabsf(v[e]) / s);
        code |= (mag | (v[e] < 0.0f && mag ? 8u : 0u)) << (4 * e);
      }
    }
    if (!on) continue;
    codes[i] = code;
    if (c % group == 0) scales[row * (kp / group) + c / group] = bad ? 0x7FC0u : (uint16_t)(__float_as_uint(s) >> 16);
  }
}

// For each weight row the power of two that takes its largest finite scale to
// [2^12, 2^13); a wave per row.
__global__ __launch_bounds__(256) void q4_unit_kernel(const uint16_t* __restrict__ scales, int n, int groups,
                                                      float* __restrict__ unit) {
  const int row = blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= n) return;
  uint32_t top = 0;  // the largest scale's exponent field
  for (int g = threadIdx.x & 63; g < groups; g += 64) {
    const uint32_t e = scales[(int64_t)row * groups + g] >> 7 & 0xFF;
    if (e < 255 && e > top) top = e;
  }
#pragma unroll
  for (int d = 32; d; d /= 2) {
    const uint32_t v = __shfl_xor(top, d);
    if (v > top) top = v;
  }
  // 2^(139 - top), it and its reciprocal kept normal numbers
  if ((threadIdx.x & 63) == 0) unit[row] = __uint_as_float((top < 13 ? 253u : 266u - top) << 23);
}

template <class T, int OUT, int GROUP>
int run_gemm_q4(GemmArgs& a, int tile, bool aligned, hipStream_t s) {
  constexpr bool PAIR = OUT == OUT_GATED;
  constexpr int KS = 64;
  if (!aligned)
    return run_gemm_tiles<T, Stage16<KS, 128, 256, 0, false, false, false>, StageQ4<T, 128, 256, GROUP, PAIR>, OUT,
                          128>(a, s);
  if (tile == 256)
    return run_gemm_tiles<T, Stage16<KS, 256, 512, 0, false, true, false>, StageQ4<T, 256, 512, GROUP, PAIR>, OUT,
                          256>(a, s);
  return run_gemm_tiles<T, Stage16<KS, 128, 256, 0, false, true, false>, StageQ4<T, 128, 256, GROUP, PAIR>, OUT,
                        128>(a, s);
}

template <class T, int OUT>
int run_gemm_q4_group(GemmArgs& a, int group, int tile, bool aligned, hipStream_t s) {
  if (group == 32) return run_gemm_q4<T, OUT, 32>(a, tile, aligned, s);
  if (group == 64) return run_gemm_q4<T, OUT, 64>(a, tile, aligned, s);
  return run_gemm_q4<T, OUT, 128>(a, tile, aligned, s);
}

GemmPlan plan_q4(const qconv_q4_desc& d, bool gated, bool aligned) {
  return gemm_plan(d.m, d.n, d.k, 1, gated, aligned, false);
}
// Of x's copy in aligned rows.
size_t copy_bytes(const qconv_q4_desc& d) { return realigns(d.k, d.ld_x, 0) ? realign_bytes(d.m, d.k) : 0; }
size_t unit_bytes(const qconv_q4_desc& d) { return (size_t)round_up(d.n, 4) * 4; }  // of one weight

int launch_gemm(const qconv_q4_desc& d, const void* x, const uint8_t* const w[2], const uint16_t* const sc[2],
                const float* bias, int act, void* y, void* ws, hipStream_t s) {
  const bool gated = w[1] != nullptr;
  GemmArgs a = {};
  a.r[0] = {(const uint16_t*)x, d.ld_x};
  a.rows = d.m;
  a.cols = d.n;
  a.k = d.k;
  a.segments = a.halves = 1;
  a.kp = (int)round_up(d.k, d.group);
  char* at = (char*)ws;
  for (int h = 0; h < (gated ? 2 : 1); ++h) {
    a.codes[h] = w[h];
    a.scales[h] = sc[h];
    if (d.dtype == QCONV_F16) {
      float* u = (float*)at;
      q4_unit_kernel<<<ceil_div(d.n, 4), 256, 0, s>>>(sc[h], d.n, a.kp / d.group, u);
      a.unit[h] = u;
      at += unit_bytes(d);
    }
  }
  if (copy_bytes(d)) {
    Realigner re(d.k, at);
    re.add(a.r[0], d.m);
    const int rc = re.run(s);
    if (rc) return rc;
    a.k = re.a.kp;  // codes past k are zero
    at += copy_bytes(d);
  }
  const bool aligned = aligned_rows(a.r[0]) && a.k % 8 == 0;
  const GemmPlan p = plan_q4(d, gated, aligned);
  a.parts = p.parts;
  a.part = (float*)at;
  a.out[0] = y;
  a.ld_out = d.ld_y;
  a.bias = bias;
  a.act = act;
  if (d.dtype == QCONV_F16)
    return gated ? run_gemm_q4_group<F16, OUT_GATED>(a, d.group, p.tile, aligned, s)
                 : run_gemm_q4_group<F16, OUT_PLAIN>(a, d.group, p.tile, aligned, s);
  return gated ? run_gemm_q4_group<BF16, OUT_GATED>(a, d.group, p.tile, aligned, s)
               : run_gemm_q4_group<BF16, OUT_PLAIN>(a, d.group, p.tile, aligned, s);
}

template <class T, int H>
int run_rows(RowsArgs& a, int group, hipStream_t s) {
  if (a.m <= FEW_MOST) {
    if (group == 32) return run_dense_few<T, 32, H>(a, s);
    if (group == 64) return run_dense_few<T, 64, H>(a, s);
    return run_dense_few<T, 128, H>(a, s);
  }
  if (group == 32) return run_dense_rows<T, Q4<32>, H>(a, s);
  if (group == 64) return run_dense_rows<T, Q4<64>, H>(a, s);
  return run_dense_rows<T, Q4<128>, H>(a, s);
}

}  // namespace

int launch_q4_pack(const void* w, int dtype, int n, int k, int64_t ld, int group, int top, uint8_t* codes,
                   uint16_t* scales, hipStream_t s) {
  const int kp = (int)round_up(k, group);
  const int64_t units = (int64_t)n * (kp / 8);
  const unsigned grid = (unsigned)(units < (1 << 22) ? (units + 255) / 256 : 1 << 14);
  uint32_t* c = (uint32_t*)codes;
  if (dtype == QCONV_F32)
    q4_pack_kernel<QCONV_F32><<<grid, 256, 0, s>>>(w, n, k, ld, group, kp, (float)top, c, scales);
  else if (dtype == QCONV_F16)
    q4_pack_kernel<QCONV_F16><<<grid, 256, 0, s>>>(w, n, k, ld, group, kp, (float)top, c, scales);
  else
    q4_pack_kernel<QCONV_BF16><<<grid, 256, 0, s>>>(w, n, k, ld, group, kp, (float)top, c, scales);
  return hip_status();
}

size_t q4_workspace_bytes(const qconv_q4_desc& d, bool gated) {
  if (d.m <= ROWS_MOST) return 0;
  const size_t u = d.dtype == QCONV_F16 ? unit_bytes(d) * (gated ? 2 : 1) : 0;
  const size_t p = plan_q4(d, gated, false).bytes, q = plan_q4(d, gated, true).bytes;
  return u + copy_bytes(d) + (p > q ? p : q);
}

int launch_q4(const qconv_q4_desc& d, const void* x, const uint8_t* w, const uint16_t* sc, const uint8_t* wu,
              const uint16_t* scu, const float* bias, int act, void* y, void* ws, hipStream_t s) {
  if (d.m == 0) return QCONV_OK;
  if (d.m > ROWS_MOST) {
    const uint8_t* const ww[2] = {w, wu};
    const uint16_t* const ss[2] = {sc, scu};
    return launch_gemm(d, x, ww, ss, bias, act, y, ws, s);
  }
  RowsArgs a = {};
  a.x = (const uint16_t*)x;
  a.ld_x = d.ld_x;
  a.ld_y = d.ld_y;
  a.w[0] = w;
  a.w[1] = wu;
  a.sc[0] = sc;
  a.sc[1] = scu;
  a.bias = bias;
  a.y = (uint16_t*)y;
  a.m = d.m;
  a.n = d.n;
  a.k = d.k;
  a.kp = (int)round_up(d.k, d.group);
  a.act = act;
  if (d.dtype == QCONV_F16) return wu ? run_rows<F16, 2>(a, d.group, s) : run_rows<F16, 1>(a, d.group, s);
  return wu ? run_rows<BF16, 2>(a, d.group, s) : run_rows<BF16, 1>(a, d.group, s);
}

}  // namespace qc
