// dense.h -- what the fully connected operators share (gated feed-forward
// block, 4-bit products): 16-bit types, the matrix instruction, activations,
// loads from any address, and the launchers behind the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/qconv.h"

namespace qc {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));

// The two 16-bit types behind one set of names: the kernels move 16-bit
// patterns and only the matrix instruction and the conversions know which.
struct F16 {
  __device__ __forceinline__ static float up(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  __device__ __forceinline__ static uint16_t down(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  // D[16 rows of a][16 rows of b] += a b^T over 32 products
  __device__ __forceinline__ static v4f mfma(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
  // the two E2M1 codes in byte BYTE of w as 16-bit values (exact)
  template <int BYTE>
  __device__ __forceinline__ static uint32_t from_e2m1(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, BYTE));
  }
  // the same times s
  template <int BYTE>
  __device__ __forceinline__ static uint32_t scaled_e2m1(uint32_t w, float s) {
    const _Float16 h = (_Float16)s;
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, BYTE) * v2h{h, h});
  }
  // For a finite bf16 scale (its bits) times `unit`: 0 if the type holds its
  // products with all magnitudes, 1 if it does together with rest_e2m1, else 2.
  // They have at most 8 + 2 significant bits, so that the smallest one decides.
  static constexpr bool REST = false;
  __device__ __forceinline__ static uint32_t odd_e2m1(uint32_t scale, float unit) {
    const float h = __uint_as_float(scale << 16) * unit * 0.5f;
    return (float)(_Float16)h == h && h != 0.0f ? 0 : 2;
  }
};
struct BF16 {
  __device__ __forceinline__ static float up(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  __device__ __forceinline__ static uint16_t down(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  __device__ __forceinline__ static v4f mfma(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  }
  template <int BYTE>
  __device__ __forceinline__ static uint32_t from_e2m1(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, BYTE));
  }
  template <int BYTE>
  __device__ __forceinline__ static uint32_t scaled_e2m1(uint32_t w, float s) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, BYTE);
    return __builtin_bit_cast(uint32_t, v2b{(__bf16)(v[0] * s), (__bf16)(v[1] * s)});
  }
  // what scaled_e2m1 has rounded away
  static constexpr bool REST = true;
  template <int BYTE>
  __device__ __forceinline__ static uint32_t rest_e2m1(uint32_t w, float s) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, BYTE);
    const float x = v[0] * s, y = v[1] * s;
    return __builtin_bit_cast(uint32_t, v2b{(__bf16)(x - (float)(__bf16)x), (__bf16)(y - (float)(__bf16)y)});
  }
  // 1.5 times a scale takes one bit more than it: 6 significant bits of 8 fit, and
  // the rest of more has 2.  2: parts of it are subnormal or 6 times it infinite.
  __device__ __forceinline__ static uint32_t odd_e2m1(uint32_t scale, float) {
    const uint32_t e = (scale >> 7) & 0xFF;
    return e - 2u > 249u ? 2 : (scale & 3) == 0 ? 0 : e >= 12 ? 1 : 2;
  }
};

// Eight 16-bit values from any 2-byte address (global loads take them).
struct __attribute__((packed, aligned(2))) U128 {
  v4u v;
};
__device__ __forceinline__ v4u load8(const uint16_t* p) { return reinterpret_cast<const U128*>(p)->v; }

// The first `n` of eight values at p, +0 for the rest; n <= 0 reads nothing.
// No byte past p[n - 1] is touched.
__device__ __forceinline__ v4u load8_first(const uint16_t* p, int n) {
  if (n >= 8) return load8(p);
  v4u r = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) r[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
  return r;
}

// 1 / (1 + exp(-g)) through the hardware's exponential and reciprocal (1 ulp
// each; the rounding of the exponent's argument adds |g| 2^-24 of exp(-g)):
// the exact division costs the tiled products' epilogue ten times as many
// instructions, and the result is rounded to 16 bits.  exp(-g) = inf gives 0.
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

// act(g) and act'(g) in fp32.  GELU's normal distribution function through erfc,
// which keeps its leading digits where g is negative: 1 + erf(g / sqrt(2))
// cancels, has 3 bits left at g = -5 and is 0 from -5.6 on.
template <int ACT>
__device__ __forceinline__ float act_value(float g) {
  if constexpr (ACT == QCONV_ACT_SILU) return g * sigmoid(g);
  else if constexpr (ACT == QCONV_ACT_GELU) return 0.5f * g * erfcf(g * -0.70710678118654752f);
  else return g < 0.0f ? 0.0f : g;  // a NaN stays
}
template <int ACT>
__device__ __forceinline__ float act_slope(float g) {
  if constexpr (ACT == QCONV_ACT_SILU) {
    const float p = sigmoid(g);
    return p * (1.0f + g * (1.0f - p));
  } else if constexpr (ACT == QCONV_ACT_GELU) {
    return 0.5f * erfcf(g * -0.70710678118654752f) + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  } else {
    return g > 0.0f ? 1.0f : 0.0f;
  }
}
// f with the activation as a constant.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == QCONV_ACT_SILU) f(std::integral_constant<int, QCONV_ACT_SILU>{});
  else if (act == QCONV_ACT_GELU) f(std::integral_constant<int, QCONV_ACT_GELU>{});
  else f(std::integral_constant<int, QCONV_ACT_RELU>{});
}
__device__ __forceinline__ float act_value(int act, float g) {
  return act == QCONV_ACT_SILU ? act_value<QCONV_ACT_SILU>(g)
                               : act == QCONV_ACT_GELU ? act_value<QCONV_ACT_GELU>(g) : act_value<QCONV_ACT_RELU>(g);
}

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

size_t ffn_forward_bytes(const qconv_ffn_desc& d);
int launch_ffn_forward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, void* h, float* pre,
                       void* ws, hipStream_t s);
size_t ffn_backward_bytes(const qconv_ffn_desc& d);
int launch_ffn_backward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, const float* pre,
                        const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s);

int launch_q4_pack(const void* w, int dtype, int n, int k, int64_t ld, int group, int top, uint8_t* codes,
                   uint16_t* scales, hipStream_t s);
size_t q4_workspace_bytes(const qconv_q4_desc& d, bool gated);
// wu / scu NULL: y = x W^T + bias; else the gated form.
int launch_q4(const qconv_q4_desc& d, const void* x, const uint8_t* w, const uint16_t* sc, const uint8_t* wu,
              const uint16_t* scu, const float* bias, int act, void* y, void* ws, hipStream_t s);

size_t grad_norm_bytes(int count, const int64_t* numel);
int launch_grad_norm(int count, const void* const* grads, const int64_t* numel, const int* dtypes, float* norm,
                     void* ws, hipStream_t s);
int launch_clip_grads(int count, const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes,
                      float max_norm, float* norm, void* ws, hipStream_t s);

}  // namespace qc
