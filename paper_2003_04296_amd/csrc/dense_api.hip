// dense_api.hip -- the C ABI of the fully connected operators and of the
// gradient norm (include/qconv.h): argument validation only.  Nothing here
// allocates or synchronises; every launch goes to the caller's stream.
#include "dense.h"

using namespace qc;

namespace {

bool half_type(int t) { return t == QCONV_F16 || t == QCONV_BF16; }
bool any_type(int t) { return t >= QCONV_F32 && t <= QCONV_BF16; }
bool group_ok(int g) { return g == 32 || g == 64 || g == 128; }
bool at(const void* p, uintptr_t align) { return ((uintptr_t)p & (align - 1)) == 0; }
constexpr int64_t MAX_LD = (int64_t)1 << 40;
constexpr int64_t MAX_NUMEL = (int64_t)1 << 38;  // 112 such tensors' pieces still count in an int

// Sizes and types of a feed-forward call.
int check_ffn(const qconv_ffn_desc* d) {
  if (!d || d->m < 0 || d->k < 1 || d->f < 1 || d->act < QCONV_ACT_SILU || d->act > QCONV_ACT_RELU)
    return QCONV_EINVAL;
  if (!any_type(d->dtype) || d->ld_x < d->k || d->ld_w < d->k || d->ld_h < d->f || d->ld_x > MAX_LD ||
      d->ld_w > MAX_LD || d->ld_h > MAX_LD)
    return QCONV_EINVAL;
  // padded sizes of every kind stay inside an int
  if (!half_type(d->dtype) || d->m > 0x7fffff00 || d->k > 0x7fffff00 || d->f > 0x3fffff00) return QCONV_EUNSUPPORTED;
  return QCONV_OK;
}

int check_q4(const qconv_q4_desc* d) {
  if (!d || d->m < 0 || d->n < 1 || d->k < 1 || !group_ok(d->group) || !any_type(d->dtype) || d->ld_x < d->k ||
      d->ld_y < d->n || d->ld_x > MAX_LD || d->ld_y > MAX_LD)
    return QCONV_EINVAL;
  if (!half_type(d->dtype) || d->m > 0x7fffff00 || d->n > 0x7fffff00 || d->k > 0x7fffff00) return QCONV_EUNSUPPORTED;
  return QCONV_OK;
}

int check_grads(int count, const void* const* grads, const int64_t* numel, const int* dtypes) {
  if (count < 0 || (count > 0 && (!grads || !numel || !dtypes))) return QCONV_EINVAL;
  for (int i = 0; i < count; ++i) {
    if (numel[i] < 0 || !any_type(dtypes[i]) || (numel[i] > 0 && !grads[i])) return QCONV_EINVAL;
    if (numel[i] > MAX_NUMEL) return QCONV_EUNSUPPORTED;
    if (!at(grads[i], dtypes[i] == QCONV_F32 ? 4 : 2)) return QCONV_EINVAL;
  }
  return QCONV_OK;
}

}  // namespace

extern "C" {

size_t qconv_ffn_pre_floats(int m, int f) {
  if (m < 0 || f < 1 || f > 0x3fffff00) return 0;
  return (size_t)m * 2 * round_up(f, 8);
}

size_t qconv_ffn_forward_bytes(const qconv_ffn_desc* d) { return check_ffn(d) ? 0 : ffn_forward_bytes(*d); }

int qconv_ffn_forward(const qconv_ffn_desc* d, const void* x, const void* w_gate, const void* w_up, void* h,
                      float* pre, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_ffn(d);
  if (rc) return rc;
  if (!w_gate || !w_up || (d->m > 0 && (!x || !h))) return QCONV_EINVAL;
  if (!at(x, 2) || !at(w_gate, 2) || !at(w_up, 2) || !at(h, 2) || !at(pre, 16) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = ffn_forward_bytes(*d);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  return launch_ffn_forward(*d, x, w_gate, w_up, h, pre, workspace, (hipStream_t)stream);
}

size_t qconv_ffn_backward_bytes(const qconv_ffn_desc* d) { return check_ffn(d) ? 0 : ffn_backward_bytes(*d); }

int qconv_ffn_backward(const qconv_ffn_desc* d, const void* x, const void* w_gate, const void* w_up,
                       const float* pre, const void* gh, void* gx, void* gw_gate, void* gw_up, void* workspace,
                       size_t workspace_bytes, void* stream) {
  const int rc = check_ffn(d);
  if (rc) return rc;
  if (!w_gate || !w_up || (d->m > 0 && (!x || !pre || !gh || !workspace)) || !gw_gate != !gw_up) return QCONV_EINVAL;
  if (!at(x, 2) || !at(w_gate, 2) || !at(w_up, 2) || !at(gh, 2) || !at(gx, 2) || !at(gw_gate, 2) || !at(gw_up, 2) ||
      !at(pre, 16) || !at(workspace, 16))
    return QCONV_EINVAL;
  if (workspace_bytes < ffn_backward_bytes(*d)) return QCONV_EWORKSPACE;
  return launch_ffn_backward(*d, x, w_gate, w_up, pre, gh, gx, gw_gate, gw_up, workspace, (hipStream_t)stream);
}

size_t qconv_q4_code_bytes(int n, int k, int group) {
  if (n < 1 || k < 1 || k > 0x7fffff00 || !group_ok(group)) return 0;
  return (size_t)n * (round_up(k, group) / 2);
}

size_t qconv_q4_scale_bytes(int n, int k, int group) {
  if (n < 1 || k < 1 || k > 0x7fffff00 || !group_ok(group)) return 0;
  return (size_t)n * (round_up(k, group) / group) * 2;
}

int qconv_q4_pack(const void* w, int dtype, int n, int k, int64_t ld_w, int group, int top, uint8_t* codes,
                  uint16_t* scales, void* stream) {
  if (!w || !codes || !scales || n < 1 || k < 1 || !any_type(dtype) || ld_w < k || ld_w > MAX_LD || !group_ok(group) ||
      (top != 4 && top != 6) || !at(w, dtype == QCONV_F32 ? 4 : 2) || !at(codes, 16) || !at(scales, 16))
    return QCONV_EINVAL;
  if (k > 0x7fffff00) return QCONV_EUNSUPPORTED;
  return launch_q4_pack(w, dtype, n, k, ld_w, group, top, codes, scales, (hipStream_t)stream);
}

size_t qconv_q4_workspace_bytes(const qconv_q4_desc* d, int gated) {
  return check_q4(d) ? 0 : q4_workspace_bytes(*d, gated != 0);
}

int qconv_q4_linear(const qconv_q4_desc* d, const void* x, const uint8_t* codes, const uint16_t* scales,
                    const float* bias, void* y, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_q4(d);
  if (rc) return rc;
  if (!codes || !scales || (d->m > 0 && (!x || !y)) || !at(x, 2) || !at(y, 2) || !at(bias, 4) || !at(codes, 16) ||
      !at(scales, 16) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = q4_workspace_bytes(*d, false);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  return launch_q4(*d, x, codes, scales, nullptr, nullptr, bias, 0, y, workspace, (hipStream_t)stream);
}

int qconv_q4_gated(const qconv_q4_desc* d, const void* x, const uint8_t* gate_codes, const uint16_t* gate_scales,
                   const uint8_t* up_codes, const uint16_t* up_scales, int act, void* y, void* workspace,
                   size_t workspace_bytes, void* stream) {
  const int rc = check_q4(d);
  if (rc) return rc;
  if (!gate_codes || !gate_scales || !up_codes || !up_scales || act < QCONV_ACT_SILU || act > QCONV_ACT_RELU ||
      (d->m > 0 && (!x || !y)) || !at(x, 2) || !at(y, 2) || !at(gate_codes, 16) || !at(gate_scales, 16) ||
      !at(up_codes, 16) || !at(up_scales, 16) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = q4_workspace_bytes(*d, true);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  return launch_q4(*d, x, gate_codes, gate_scales, up_codes, up_scales, nullptr, act, y, workspace,
                   (hipStream_t)stream);
}

size_t aqe_grad_norm_bytes(int count, const int64_t* numel) {
  if (count < 1 || !numel) return 0;
  for (int i = 0; i < count; ++i)
    if (numel[i] < 0) return 0;
  return grad_norm_bytes(count, numel);
}

int aqe_grad_norm(int count, const void* const* grads, const int64_t* numel, const int* dtypes, float* norm,
                  void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_grads(count, grads, numel, dtypes);
  if (rc) return rc;
  if (!norm || !at(norm, 4) || !at(workspace, 16)) return QCONV_EINVAL;
  const size_t need = aqe_grad_norm_bytes(count, numel);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  return launch_grad_norm(count, grads, numel, dtypes, norm, workspace, (hipStream_t)stream);
}

int aqe_clip_grads(int count, const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes,
                   float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_grads(count, grads, numel, dtypes);
  if (rc) return rc;
  if (!norm || !at(norm, 4) || !at(workspace, 16) || (count > 0 && !out) || !(max_norm >= 0.0f)) return QCONV_EINVAL;
  for (int i = 0; i < count; ++i)
    if ((numel[i] > 0 && !out[i]) || !at(out[i], dtypes[i] == QCONV_F32 ? 4 : 2)) return QCONV_EINVAL;
  const size_t need = aqe_grad_norm_bytes(count, numel);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  return launch_clip_grads(count, grads, out, numel, dtypes, max_norm, norm, workspace, (hipStream_t)stream);
}

}  // extern "C"
