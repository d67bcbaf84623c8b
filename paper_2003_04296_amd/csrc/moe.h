// moe.h -- launchers of the operators for rows that go to different weights:
// the rows' order, the experts' products and low-rank adapters.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/qconv.h"

namespace qc {

constexpr int MOE_GROUPS_MOST = 4096;

size_t moe_sort_bytes(int n, int groups);
int launch_moe_sort(const void* ids, int wide, int tokens, int slots, int64_t ld, int groups, int* offsets, int* order,
                    int* place, void* ws, hipStream_t s);
int launch_moe_gather(const qconv_moe_rows_desc& d, const void* x, const int* place, void* rows, hipStream_t s);
int launch_moe_combine(const qconv_moe_rows_desc& d, const void* ys, const int* place, const float* weights, void* y,
                       hipStream_t s);
int launch_moe_combine_back(const qconv_moe_rows_desc& d, const void* gy, const void* ys, const int* place,
                            const float* weights, void* gys, int64_t ld_gys, float* gw, hipStream_t s);

size_t moe_forward_bytes(const qconv_moe_desc& d, bool gated);
// wu NULL: the linear form.
int launch_moe_forward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                       void* h, float* pre, void* ws, hipStream_t s);
size_t moe_backward_bytes(const qconv_moe_desc& d, bool gated);
int launch_moe_backward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                        const float* pre, const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s);

size_t lora_forward_bytes(const qconv_lora_desc& d, bool keep_mid);
int launch_lora_forward(const qconv_lora_desc& d, const void* x, const void* wa, const void* wb, const int* offsets,
                        const int* order, const float* scale, const void* y, void* out, float* mid, void* ws,
                        hipStream_t s);
size_t lora_backward_bytes(const qconv_lora_desc& d);
int launch_lora_backward(const qconv_lora_desc& d, const void* x, const void* wa, const void* wb, const int* offsets,
                         const int* order, const float* scale, const float* mid, const void* gy, void* gx, void* ga,
                         void* gb, void* ws, hipStream_t s);

}  // namespace qc
