// dense_ffn.h -- what the gated block of one weight and that of many experts
// share beside the tiles: the products' factors in the backward pass.
#pragma once

#include "dense_gemm.h"

namespace qc {

// dg and du of four hidden features per thread, into [m][2][fp] with the
// columns past f zero (gx's products run over all fp of them).  They are
// rounded to the tensors' type, once, because the matrix cores take 16-bit
// operands; g and u themselves stay in fp32 between the passes.  The gradients'
// error is 1.4 times that of fp32 factors (two roundings in place of one), and a
// factor past fp16's 65504 is infinite, as a gradient of that type is.  Two parts
// per factor would hold both and double the backward's products.  Bound by HBM:
// 8192 tokens of 16384 features read 1.3 GB and write 0.5 in 352 us, 5.3 TB/s.
// count: the rows there are, where only the device knows (at most m), or NULL.
template <class T, int ACT>
static __global__ __launch_bounds__(256) void ffn_slopes_kernel(const float* __restrict__ pre, const uint16_t* __restrict__ gh,
                                                         int64_t ld_h, int m, int f, int fp, const int* count,
                                                         uint16_t* __restrict__ d) {
  if (count) m = *count < m ? *count : m;
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

template <class T>
int run_slopes(int act, const float* pre, const void* gh, int64_t ld_h, int m, int f, const int* count, uint16_t* out,
               hipStream_t s) {
  const int fp = (int)round_up(f, 8);
  const int64_t n = (int64_t)m * (fp / 4);
  const unsigned grid = (unsigned)(n < (1 << 23) ? (n + 255) / 256 : 1 << 15);
  const uint16_t* g = (const uint16_t*)gh;
  if (act == QCONV_ACT_SILU)
    ffn_slopes_kernel<T, QCONV_ACT_SILU><<<grid, 256, 0, s>>>(pre, g, ld_h, m, f, fp, count, out);
  else if (act == QCONV_ACT_GELU)
    ffn_slopes_kernel<T, QCONV_ACT_GELU><<<grid, 256, 0, s>>>(pre, g, ld_h, m, f, fp, count, out);
  else
    ffn_slopes_kernel<T, QCONV_ACT_RELU><<<grid, 256, 0, s>>>(pre, g, ld_h, m, f, fp, count, out);
  return hip_status();
}

}  // namespace qc
