// moe_api.hip -- the C ABI of the operators for rows that go to different
// weights (include/qconv.h): argument validation only.  Nothing here allocates or
// synchronises; every launch goes to the caller's stream.
#include <initializer_list>

#include "dense.h"
#include "moe.h"

using namespace qc;

namespace {

bool half_type(int t) { return t == QCONV_F16 || t == QCONV_BF16; }
bool any_type(int t) { return t >= QCONV_F32 && t <= QCONV_BF16; }
bool at(const void* p, uintptr_t align) { return ((uintptr_t)p & (align - 1)) == 0; }
constexpr int64_t MAX_LD = (int64_t)1 << 40;
constexpr int MOST = 0x7fffff00;  // padded sizes of every kind stay inside an int

static_assert(QCONV_MOE_GROUPS_MOST == MOE_GROUPS_MOST, "one limit");

int check_groups(int groups) {
  if (groups < 1) return QCONV_EINVAL;
  return groups > MOE_GROUPS_MOST ? QCONV_EUNSUPPORTED : QCONV_OK;
}

int check_sort(int tokens, int slots, int groups) {
  if (tokens < 0 || slots < 1) return QCONV_EINVAL;
  if ((int64_t)tokens * slots > MOST) return QCONV_EUNSUPPORTED;
  return check_groups(groups);
}

int check_rows(const qconv_moe_rows_desc* d) {
  if (!d || d->tokens < 0 || d->slots < 1 || d->width < 1 || !any_type(d->dtype) || d->ld_tokens < d->width ||
      d->ld_rows < d->width || d->ld_tokens > MAX_LD || d->ld_rows > MAX_LD)
    return QCONV_EINVAL;
  if ((int64_t)d->tokens * d->slots > MOST || d->width > MOST) return QCONV_EUNSUPPORTED;
  return QCONV_OK;
}

int check_moe(const qconv_moe_desc* d) {
  if (!d || d->rows < 0 || d->k < 1 || d->f < 1 || d->act < QCONV_ACT_SILU || d->act > QCONV_ACT_RELU ||
      !any_type(d->dtype) || d->ld_x < d->k || d->ld_w < d->k || d->ld_h < d->f || d->ld_x > MAX_LD ||
      d->ld_w > MAX_LD || d->ld_h > MAX_LD)
    return QCONV_EINVAL;
  const int rc = check_groups(d->groups);
  if (rc) return rc;
  if (!half_type(d->dtype) || d->rows > MOST || d->k > MOST || d->f > 0x3fffff00) return QCONV_EUNSUPPORTED;
  return QCONV_OK;
}

// Where a tensor lies: rows of `len` bytes, `ld` apart.
struct Span {
  uintptr_t p;
  uint64_t rows, ld, len;
};
Span rows_at(const void* p, int64_t rows, int64_t ld, int64_t cols, int size) {
  return {(uintptr_t)p, p ? (uint64_t)rows : 0, (uint64_t)ld * size, (uint64_t)cols * size};
}
Span block_at(const void* p, int64_t values, int size) { return rows_at(p, values > 0 ? 1 : 0, values, values, size); }
// Whether two tensors share a byte.  Those whose rows lie between the other's do not.
bool cross(Span a, Span b) {
  if (a.rows == 0 || b.rows == 0) return false;
  if (b.p < a.p) {
    const Span t = a;
    a = b;
    b = t;
  }
  uint64_t d = b.p - a.p;
  for (uint64_t i = 0; i < b.rows; ++i, d += b.ld) {
    const uint64_t row = d / a.ld, in = d % a.ld;
    if (row >= a.rows) return false;
    if (in < a.len) return true;
    if (row + 1 == a.rows) return false;
    if (b.len > a.ld - in) return true;
    if (b.ld == a.ld) return false;  // the further rows lie as this one
  }
  return false;
}
bool cross(const Span& a, std::initializer_list<Span> others) {
  for (const Span& b : others)
    if (cross(a, b)) return true;
  return false;
}
Span weights_at(const qconv_moe_desc* d, const void* w) { return rows_at(w, (int64_t)d->groups * d->f, d->ld_w, d->k, 2); }
Span weight_grads_at(const qconv_moe_desc* d, const void* gw) { return block_at(gw, (int64_t)d->groups * d->f * d->k, 2); }

// What both forms of the experts' products have in common.
int check_forward(const qconv_moe_desc* d, const void* x, const void* w, const void* w_up, const int32_t* offsets,
                  const void* h, const float* pre, const void* workspace, size_t workspace_bytes) {
  if (!w || !offsets || (d->rows > 0 && (!x || !h)) || !at(x, 2) || !at(w, 2) || !at(h, 2) || !at(offsets, 4) ||
      !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = moe_forward_bytes(*d, w_up);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  const Span rows = rows_at(x, d->rows, d->ld_x, d->k, 2), from = block_at(offsets, d->groups + 1, 4);
  const Span to = rows_at(h, d->rows, d->ld_h, d->f, 2);
  const Span kept = block_at(pre, (int64_t)qconv_ffn_pre_floats(d->rows, d->f), 4);
  const Span wg = weights_at(d, w), wu = weights_at(d, w_up);
  return cross(to, {rows, from, wg, wu, kept}) || cross(kept, {rows, from, wg, wu}) ? QCONV_EINVAL : QCONV_OK;
}
// The gradient of x is written first, the weights' are next; the gated form is done with
// gh and pre by then.
int check_backward(const qconv_moe_desc* d, const void* x, const void* w, const void* w_up, const int32_t* offsets,
                   const void* gh, const void* gx, const void* gw, const void* gw_up, const void* workspace,
                   size_t workspace_bytes) {
  if (!w || !offsets || (d->rows > 0 && (!x || !gh)) || !at(x, 2) || !at(w, 2) || !at(gh, 2) || !at(gx, 2) ||
      !at(gw, 2) || !at(offsets, 4) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = moe_backward_bytes(*d, w_up);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  const Span rows = rows_at(gw ? x : nullptr, d->rows, d->ld_x, d->k, 2), from = block_at(offsets, d->groups + 1, 4);
  const Span grads = rows_at(w_up ? nullptr : gh, d->rows, d->ld_h, d->f, 2);
  const Span to = block_at(gx, (int64_t)d->rows * d->k, 2);
  for (const void* g : {gw, gw_up})
    if (cross(weight_grads_at(d, g), {rows, from, grads, to, weight_grads_at(d, g == gw ? gw_up : nullptr)})) return QCONV_EINVAL;
  return cross(to, {rows, from, grads, weights_at(d, w), weights_at(d, w_up)}) ? QCONV_EINVAL : QCONV_OK;
}

int check_lora(const qconv_lora_desc* d, bool out) {
  if (!d || d->m < 0 || d->rank < 1 || d->k < 1 || d->n < 1 || !any_type(d->dtype) || d->ld_x < d->k ||
      d->ld_y < d->n || (out && d->ld_out < d->n) || d->ld_x > MAX_LD || d->ld_y > MAX_LD || (out && d->ld_out > MAX_LD))
    return QCONV_EINVAL;
  const int rc = check_groups(d->groups);
  if (rc) return rc;
  if (!half_type(d->dtype) || d->rank > QCONV_LORA_RANK_MOST || d->m > MOST || d->k > MOST || d->n > MOST)
    return QCONV_EUNSUPPORTED;
  return QCONV_OK;
}
// Adapters, their tokens and scales.
bool lora_inputs(const qconv_lora_desc* d, const void* x, const void* a, const void* b, const int32_t* offsets,
                 const int32_t* order, const float* scale, const void* y) {
  return a && b && offsets && (d->m == 0 || (x && order && y)) && at(x, 2) && at(a, 2) && at(b, 2) && at(y, 2) &&
         at(offsets, 4) && at(order, 4) && at(scale, 4);
}

}  // namespace

extern "C" {

size_t qconv_moe_sort_bytes(int tokens, int slots, int groups) {
  return check_sort(tokens, slots, groups) ? 0 : moe_sort_bytes(tokens * slots, groups);
}

int qconv_moe_sort(const void* ids, int wide, int tokens, int slots, int64_t ld, int groups, int32_t* offsets,
                   int32_t* order, int32_t* place, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_sort(tokens, slots, groups);
  if (rc) return rc;
  if (!offsets || (tokens > 0 && (!ids || !order || !place)) || ld < slots || ld > MAX_LD || !at(ids, wide ? 8 : 4) ||
      !at(offsets, 4) || !at(order, 4) || !at(place, 4) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = moe_sort_bytes(tokens * slots, groups);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  // a value of place is written after the last read of its id
  const Span from = rows_at(ids, tokens, ld, slots, wide ? 8 : 4);
  const bool over = place == ids && !wide && ld == slots;
  if (cross(from, {block_at(offsets, groups + 1, 4), block_at(order, (int64_t)tokens * slots, 4),
                   block_at(over ? nullptr : place, (int64_t)tokens * slots, 4)}))
    return QCONV_EINVAL;
  return launch_moe_sort(ids, wide != 0, tokens, slots, ld, groups, offsets, order, place, workspace,
                         (hipStream_t)stream);
}

int qconv_moe_gather(const qconv_moe_rows_desc* d, const void* x, const int32_t* place, void* rows, void* stream) {
  const int rc = check_rows(d);
  if (rc) return rc;
  const int a = d->dtype == QCONV_F32 ? 4 : 2;
  if ((d->tokens > 0 && (!x || !place || !rows)) || !at(x, a) || !at(rows, a) || !at(place, 4)) return QCONV_EINVAL;
  const int64_t n = (int64_t)d->tokens * d->slots;
  if (cross(rows_at(rows, n, d->ld_rows, d->width, a), {rows_at(x, d->tokens, d->ld_tokens, d->width, a), block_at(place, n, 4)}))
    return QCONV_EINVAL;
  return launch_moe_gather(*d, x, place, rows, (hipStream_t)stream);
}

int qconv_moe_combine(const qconv_moe_rows_desc* d, const void* rows, const int32_t* place, const float* weights,
                      void* y, void* stream) {
  const int rc = check_rows(d);
  if (rc) return rc;
  const int a = d->dtype == QCONV_F32 ? 4 : 2;
  if ((d->tokens > 0 && (!rows || !place || !y)) || !at(rows, a) || !at(y, a) || !at(place, 4) || !at(weights, 4))
    return QCONV_EINVAL;
  const int64_t n = (int64_t)d->tokens * d->slots;
  if (cross(rows_at(y, d->tokens, d->ld_tokens, d->width, a),
            {rows_at(rows, n, d->ld_rows, d->width, a), block_at(place, n, 4), block_at(weights, n, 4)}))
    return QCONV_EINVAL;
  return launch_moe_combine(*d, rows, place, weights, y, (hipStream_t)stream);
}

int qconv_moe_combine_backward(const qconv_moe_rows_desc* d, const void* gy, const void* rows, const int32_t* place,
                               const float* weights, void* grows, int64_t ld_grows, float* gweights, void* stream) {
  const int rc = check_rows(d);
  if (rc) return rc;
  const int a = d->dtype == QCONV_F32 ? 4 : 2;
  if ((d->tokens > 0 && (!gy || !place || (gweights && !rows))) || (grows && (ld_grows < d->width || ld_grows > MAX_LD)) ||
      !at(gy, a) || !at(rows, a) || !at(grows, a) || !at(place, 4) || !at(weights, 4) || !at(gweights, 4))
    return QCONV_EINVAL;
  // a value of rows, and a weight, is read before the gradient in its place is written
  const int64_t n = (int64_t)d->tokens * d->slots;
  const Span token = rows_at(gy, d->tokens, d->ld_tokens, d->width, a), places = block_at(place, n, 4);
  const Span expert = rows_at(gweights ? rows : nullptr, n, d->ld_rows, d->width, a), w = block_at(weights, n, 4);
  const Span to = rows_at(grows, n, ld_grows, d->width, a), to_w = block_at(gweights, n, 4);
  if (cross(to, {token, places, w}) || (!(grows == rows && ld_grows == d->ld_rows) && cross(to, expert)) ||
      cross(to_w, {token, places, expert, to}) || (gweights != weights && cross(to_w, w)))
    return QCONV_EINVAL;
  return launch_moe_combine_back(*d, gy, rows, place, weights, grows, ld_grows, gweights, (hipStream_t)stream);
}

size_t qconv_moe_forward_bytes(const qconv_moe_desc* d, int gated) {
  return check_moe(d) ? 0 : moe_forward_bytes(*d, gated != 0);
}

int qconv_moe_gated_forward(const qconv_moe_desc* d, const void* x, const void* w_gate, const void* w_up,
                            const int32_t* offsets, void* h, float* pre, void* workspace, size_t workspace_bytes,
                            void* stream) {
  int rc = check_moe(d);
  if (rc) return rc;
  if (!w_up || !at(w_up, 2) || !at(pre, 16)) return QCONV_EINVAL;
  rc = check_forward(d, x, w_gate, w_up, offsets, h, pre, workspace, workspace_bytes);
  return rc ? rc : launch_moe_forward(*d, x, w_gate, w_up, offsets, h, pre, workspace, (hipStream_t)stream);
}

int qconv_moe_linear_forward(const qconv_moe_desc* d, const void* x, const void* w, const int32_t* offsets, void* y,
                             void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_moe(d);
  if (rc) return rc;
  rc = check_forward(d, x, w, nullptr, offsets, y, nullptr, workspace, workspace_bytes);
  return rc ? rc : launch_moe_forward(*d, x, w, nullptr, offsets, y, nullptr, workspace, (hipStream_t)stream);
}

size_t qconv_moe_backward_bytes(const qconv_moe_desc* d, int gated) {
  return check_moe(d) ? 0 : moe_backward_bytes(*d, gated != 0);
}

int qconv_moe_gated_backward(const qconv_moe_desc* d, const void* x, const void* w_gate, const void* w_up,
                             const int32_t* offsets, const float* pre, const void* gh, void* gx, void* gw_gate,
                             void* gw_up, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_moe(d);
  if (rc) return rc;
  if (!w_up || (d->rows > 0 && !pre) || !gw_gate != !gw_up || !at(w_up, 2) || !at(gw_up, 2) || !at(pre, 16))
    return QCONV_EINVAL;
  rc = check_backward(d, x, w_gate, w_up, offsets, gh, gx, gw_gate, gw_up, workspace, workspace_bytes);
  return rc ? rc : launch_moe_backward(*d, x, w_gate, w_up, offsets, pre, gh, gx, gw_gate, gw_up, workspace,
                                       (hipStream_t)stream);
}

int qconv_moe_linear_backward(const qconv_moe_desc* d, const void* x, const void* w, const int32_t* offsets,
                              const void* gy, void* gx, void* gw, void* workspace, size_t workspace_bytes,
                              void* stream) {
  int rc = check_moe(d);
  if (rc) return rc;
  rc = check_backward(d, x, w, nullptr, offsets, gy, gx, gw, nullptr, workspace, workspace_bytes);
  return rc ? rc : launch_moe_backward(*d, x, w, nullptr, offsets, nullptr, gy, gx, gw, nullptr, workspace,
                                       (hipStream_t)stream);
}

size_t qconv_lora_mid_floats(int m, int rank) {
  if (m < 0 || rank < 1 || rank > QCONV_LORA_RANK_MOST) return 0;
  return (size_t)m * round_up(rank, 4);
}

size_t qconv_lora_forward_bytes(const qconv_lora_desc* d, int keep_mid) {
  return check_lora(d, true) ? 0 : lora_forward_bytes(*d, keep_mid != 0);
}

int qconv_lora_forward(const qconv_lora_desc* d, const void* x, const void* a, const void* b, const int32_t* offsets,
                       const int32_t* order, const float* scale, const void* y, void* out, float* mid,
                       void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_lora(d, true);
  if (rc) return rc;
  if (!lora_inputs(d, x, a, b, offsets, order, scale, y) || (d->m > 0 && !out) || !at(out, 2) || !at(mid, 16) ||
      !at(workspace, 16) || (out && out == y && d->ld_out != d->ld_y))
    return QCONV_EINVAL;
  const size_t need = lora_forward_bytes(*d, mid != nullptr);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  // one launch for few tokens reads a row of x in every block of the result's columns
  const Span to = rows_at(out, d->m, d->ld_out, d->n, 2);
  if (cross(to, {rows_at(x, d->m, d->ld_x, d->k, 2), rows_at(out == y ? nullptr : y, d->m, d->ld_y, d->n, 2),
                 block_at(a, (int64_t)d->groups * d->rank * d->k, 2), block_at(b, (int64_t)d->groups * d->n * d->rank, 2),
                 block_at(offsets, d->groups + 1, 4), block_at(order, d->m, 4), block_at(scale, d->groups, 4),
                 block_at(mid, (int64_t)qconv_lora_mid_floats(d->m, d->rank), 4)}))
    return QCONV_EINVAL;
  return launch_lora_forward(*d, x, a, b, offsets, order, scale, y, out, mid, workspace, (hipStream_t)stream);
}

size_t qconv_lora_backward_bytes(const qconv_lora_desc* d) { return check_lora(d, false) ? 0 : lora_backward_bytes(*d); }

int qconv_lora_backward(const qconv_lora_desc* d, const void* x, const void* a, const void* b, const int32_t* offsets,
                        const int32_t* order, const float* scale, const float* mid, const void* gy, void* gx, void* ga,
                        void* gb, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_lora(d, false);
  if (rc) return rc;
  if (!lora_inputs(d, x, a, b, offsets, order, scale, gy) || !ga != !gb || (d->m > 0 && ga && !mid) || !at(gx, 2) ||
      !at(ga, 2) || !at(gb, 2) || !at(mid, 16) || !at(workspace, 16))
    return QCONV_EINVAL;
  const size_t need = lora_backward_bytes(*d);
  if (need && !workspace) return QCONV_EINVAL;
  if (workspace_bytes < need) return QCONV_EWORKSPACE;
  // gx is written first, then ga, then gb; a and b have been copied by then
  const Span rows = rows_at(ga ? x : nullptr, d->m, d->ld_x, d->k, 2), grads = rows_at(ga ? gy : nullptr, d->m, d->ld_y, d->n, 2);
  const Span from = block_at(offsets, d->groups + 1, 4), tokens = block_at(order, d->m, 4), scales = block_at(scale, d->groups, 4);
  const Span kept = block_at(ga ? mid : nullptr, (int64_t)qconv_lora_mid_floats(d->m, d->rank), 4);
  const Span to = block_at(gx, (int64_t)d->m * d->k, 2), to_a = block_at(ga, (int64_t)d->groups * d->rank * d->k, 2);
  const Span to_b = block_at(gb, (int64_t)d->groups * d->n * d->rank, 2);
  if (cross(to, {rows, grads, from, tokens, scales, kept, to_a, to_b}) ||
      cross(to_a, {rows, grads, from, tokens, scales, kept, to_b}) || cross(to_b, {grads, from, tokens, scales, kept}))
    return QCONV_EINVAL;
  return launch_lora_backward(*d, x, a, b, offsets, order, scale, mid, gy, gx, ga, gb, workspace, (hipStream_t)stream);
}

}  // extern "C"
