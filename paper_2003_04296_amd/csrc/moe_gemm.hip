// moe_gemm.hip -- the experts' products: rows offsets[e] .. offsets[e + 1] of x
// with the weights of expert e, forward and backward, in 16-bit types.
//   gated    h = act(x Wg_e^T) (x Wu_e^T), as ffn.hip for each expert's rows
//   linear   y = x W_e^T;  gx = gy W_e;  gW_e = gy_e^T x_e
// One launch per product for all experts, on the tiles of dense_gemm.h: a block
// finds its expert and rows from the offsets, which stay on the device.
#include "dense_ffn.h"
#include "moe.h"
#include "moe_groups.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// The products whose rows are the batch's (forward, gx).
template <class T, class SR, class SC, int OUT, int B>
__global__ __launch_bounds__(B / 64 * 128) void moe_gemm_kernel(GemmArgs a, Groups g, int64_t step_c) {
  [[maybe_unused]] __shared__ v4u lds[STAGES<SR::KS> * (B + B) * SR::CPR];
#ifdef __HIP_DEVICE_COMPILE__  // the host has no LDS pointers
  const GroupPieces pieces(g, B);
  if (blockIdx.x >= (uint64_t)pieces.total * a.tiles_c) return;
  TileAt at = tile_at(blockIdx.x, pieces.total, a.tiles_c);
  int e, piece;
  pieces.find(g, at.r, e, piece);
  const GroupRows rows = group_rows(g, e);
  const int64_t first = __builtin_amdgcn_readfirstlane(rows.first);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a.r[i].p += first * a.r[i].ld;
    a.c[i].p += e * step_c;
  }
  a.rows = __builtin_amdgcn_readfirstlane(rows.count);
  a.out[0] = (uint16_t*)a.out[0] + first * a.ld_out;
  if (OUT == OUT_GATED && a.pre) a.pre += first * 2 * a.ld_pre;
  at.r = piece;
  a.tiles_r = 0x7fffffff;  // one half
  gemm_tile<T, SR, SC, OUT, B, B>(a, (lds_v4u*)lds, at, 0);
#endif
}

// The products over the batch's rows (weight gradients): a.rows and a.cols are
// the weight's.
template <class T, class SR, class SC, int B>
__global__ __launch_bounds__(B / 64 * 128) void moe_gemm_w_kernel(GemmArgs a, Groups g, int64_t step_out) {
  [[maybe_unused]] __shared__ v4u lds[STAGES<SR::KS> * (B + B) * SR::CPR];
#ifdef __HIP_DEVICE_COMPILE__
  // one expert after the other, each over all dies: the experts' sums differ in length
  const uint32_t per = a.tiles_r * a.halves, all = per * a.tiles_c;
  const int e = blockIdx.x / all;
  const TileAt at = tile_at(blockIdx.x % all, per, a.tiles_c);
  const GroupRows rows = group_rows(g, e);
  const int64_t first = __builtin_amdgcn_readfirstlane(rows.first);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a.r[i].p += first * a.r[i].ld;
    a.out[i] = (uint16_t*)a.out[i] + e * step_out;
  }
  a.c[0].p += first * a.c[0].ld;
  a.k = __builtin_amdgcn_readfirstlane(rows.count);
  gemm_tile<T, SR, SC, OUT_PLAIN, B, B>(a, (lds_v4u*)lds, at, 0);
#endif
}

template <class T, class SR, class SC, int OUT, int B>
int run_tiles(GemmArgs& a, const Groups& g, int64_t step_c, hipStream_t s) {
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? B / 2 : B);
  const int64_t blocks = GroupPieces::most(g.rows, g.n, B) * a.tiles_c;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  a.wide_out = a.ld_out % 4 == 0 && ((uintptr_t)a.out[0] & 7) == 0;
  moe_gemm_kernel<T, SR, SC, OUT, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a, g, step_c);
  return hip_status();
}
template <class T, class SR, class SC, int B>
int run_tiles_w(GemmArgs& a, const Groups& g, int64_t step_out, hipStream_t s) {
  a.tiles_r = ceil_div(a.rows, B);
  a.tiles_c = ceil_div(a.cols, B);
  const int64_t blocks = (int64_t)a.tiles_r * a.halves * a.tiles_c * g.n;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;
  a.wide_out = a.ld_out % 4 == 0 && ((uintptr_t)a.out[0] & 7) == 0 && ((uintptr_t)a.out[1] & 7) == 0;
  moe_gemm_w_kernel<T, SR, SC, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a, g, step_out);
  return hip_status();
}

// Rows of the batch by the weights' rows (CCOL false) or columns.
template <class T, bool CCOL, int OUT>
int run_rows_t(GemmArgs& a, const Groups& g, int64_t step_c, int tile, bool aligned, hipStream_t s) {
  constexpr bool PAIR = OUT == OUT_GATED;
  constexpr int KS = CCOL ? 32 : 64;
  if (!aligned)
    return run_tiles<T, Stage16<KS, 128, 256, 0, false, false, false>, Stage16<KS, 128, 256, 1, CCOL, false, PAIR>, OUT,
                     128>(a, g, step_c, s);
  if (tile == 256)
    return run_tiles<T, Stage16<KS, 256, 512, 0, false, true, false>, Stage16<KS, 256, 512, 1, CCOL, true, PAIR>, OUT,
                     256>(a, g, step_c, s);
  return run_tiles<T, Stage16<KS, 128, 256, 0, false, true, false>, Stage16<KS, 128, 256, 1, CCOL, true, PAIR>, OUT,
                   128>(a, g, step_c, s);
}
template <bool CCOL, int OUT>
int run_rows(int dtype, GemmArgs& a, const Groups& g, int64_t step_c, int tile, bool aligned, hipStream_t s) {
  return dtype == QCONV_F16 ? run_rows_t<F16, CCOL, OUT>(a, g, step_c, tile, aligned, s)
                            : run_rows_t<BF16, CCOL, OUT>(a, g, step_c, tile, aligned, s);
}
template <class T>
int run_weights_t(GemmArgs& a, const Groups& g, int64_t step_out, int tile, bool aligned, hipStream_t s) {
  if (!aligned)
    return run_tiles_w<T, Stage16<32, 128, 256, 0, true, false, false>, Stage16<32, 128, 256, 1, true, false, false>,
                       128>(a, g, step_out, s);
  if (tile == 256)
    return run_tiles_w<T, Stage16<32, 256, 512, 0, true, true, false>, Stage16<32, 256, 512, 1, true, true, false>,
                       256>(a, g, step_out, s);
  return run_tiles_w<T, Stage16<32, 128, 256, 0, true, true, false>, Stage16<32, 128, 256, 1, true, true, false>, 128>(
      a, g, step_out, s);
}

// Tiles of 256 x 256 where the experts' rows fill most of them and there are
// enough for the 256 compute units, else 128 x 128.
int tile_rows(const qconv_moe_desc& d, int cols, bool gated) {
  const int64_t across = gated ? 128 : 256;
  return d.rows >= 512 * (int64_t)d.groups && d.rows / 256 * ((cols + across - 1) / across) >= 256 ? 256 : 128;
}
int tile_weights(const qconv_moe_desc& d, int halves) {
  return (int64_t)ceil_div(d.f, 256) * ceil_div(d.k, 256) * halves * d.groups >= 256 ? 256 : 128;
}

// Operands off 16-byte rows are copied as in ffn.hip; the copies of all experts'
// weights pay from so many rows an expert on.
constexpr int COPY_LEAST = 384;
int64_t fp_of(const qconv_moe_desc& d) { return round_up(d.f, 8); }
size_t copies_bytes(const qconv_moe_desc& d, bool gated, bool forward) {
  if (forward && d.rows < COPY_LEAST * (int64_t)d.groups) return 0;
  return realigns(d.k, d.ld_x, d.ld_w)
             ? realign_bytes(d.rows, d.k) + (gated ? 2 : 1) * realign_bytes((int64_t)d.groups * d.f, d.k)
             : 0;
}
// The factors of the backward's products: dg and du, or a copy of gy where its
// rows are off 16 bytes.
size_t factor_bytes(const qconv_moe_desc& d, bool gated) {
  if (!gated) return realigns(d.f, d.ld_h, d.ld_h) ? realign_bytes(d.rows, d.f) : 0;
  return (size_t)round_up((int64_t)d.rows * 2 * fp_of(d) * 2, 16);
}

}  // namespace

size_t moe_forward_bytes(const qconv_moe_desc& d, bool gated) { return copies_bytes(d, gated, true); }

int launch_moe_forward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                       void* h, float* pre, void* ws, hipStream_t s) {
  if (d.rows == 0) return QCONV_OK;
  const Groups g = {offsets, d.groups, d.rows};
  GemmArgs a = {};
  a.r[0] = a.r[1] = {(const uint16_t*)x, d.ld_x};
  a.c[0] = {(const uint16_t*)wg, d.ld_w};
  a.c[1] = wu ? Operand{(const uint16_t*)wu, d.ld_w} : a.c[0];
  a.cols = d.f;
  a.k = d.k;
  a.segments = a.halves = a.parts = 1;
  a.out[0] = h;
  a.ld_out = d.ld_h;
  a.pre = pre;
  a.ld_pre = (int)round_up(d.f, 8);
  a.act = d.act;
  if (copies_bytes(d, wu, true)) {
    Realigner re(d.k, ws);
    re.add(a.r[0], d.rows);
    if (wu) {
      re.add_pair(a.c[0], a.c[1], (int64_t)d.groups * d.f);
    } else {
      re.add(a.c[0], (int64_t)d.groups * d.f);
      a.c[1] = a.c[0];
    }
    a.r[1] = a.r[0];
    const int rc = re.run(s);
    if (rc) return rc;
    a.k = re.a.kp;
  }
  const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && aligned_rows(a.c[1]) && a.k % 8 == 0;
  const int64_t step = (int64_t)d.f * a.c[0].ld;
  if (wu) return run_rows<false, OUT_GATED>(d.dtype, a, g, step, tile_rows(d, d.f, true), aligned, s);
  return run_rows<false, OUT_PLAIN>(d.dtype, a, g, step, tile_rows(d, d.f, false), aligned, s);
}

size_t moe_backward_bytes(const qconv_moe_desc& d, bool gated) {
  return copies_bytes(d, gated, false) + factor_bytes(d, gated);
}

int launch_moe_backward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                        const float* pre, const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s) {
  const Groups g = {offsets, d.groups, d.rows};
  const int fp = (int)round_up(d.f, 8);
  Operand ox = {(const uint16_t*)x, d.ld_x}, og = {(const uint16_t*)wg, d.ld_w};
  Operand ou = wu ? Operand{(const uint16_t*)wu, d.ld_w} : og;
  uint16_t* factors = (uint16_t*)((char*)ws + copies_bytes(d, wu, false));
  bool whole = d.k % 8 == 0;  // rows end with 16 bytes
  int rc = QCONV_OK;
  if (copies_bytes(d, wu, false)) {
    Realigner re(d.k, ws);
    if (gwg) re.add(ox, d.rows);
    if (gx && d.rows > 0) {
      if (wu) {
        re.add_pair(og, ou, (int64_t)d.groups * d.f);
      } else {
        re.add(og, (int64_t)d.groups * d.f);
        ou = og;
      }
    }
    rc = re.run(s);
    if (rc) return rc;
    whole = true;
  }
  Operand d0, d1;
  bool whole_h = true;
  if (wu) {
    d0 = {factors, 2 * (int64_t)fp};
    d1 = {factors + fp, 2 * (int64_t)fp};
    if (d.rows > 0)
      rc = d.dtype == QCONV_F16 ? run_slopes<F16>(d.act, pre, gh, d.ld_h, d.rows, d.f, offsets + d.groups, factors, s)
                                : run_slopes<BF16>(d.act, pre, gh, d.ld_h, d.rows, d.f, offsets + d.groups, factors, s);
  } else {
    d0 = {(const uint16_t*)gh, d.ld_h};
    if (factor_bytes(d, false)) {
      Realigner re(d.f, factors);
      re.add(d0, d.rows);
      rc = re.run(s);
    } else {
      whole_h = d.f % 8 == 0;
    }
    d1 = d0;
  }
  if (rc == QCONV_OK && gx && d.rows > 0) {
    GemmArgs a = {};
    a.r[0] = d0;
    a.r[1] = d1;
    a.c[0] = og;
    a.c[1] = ou;
    a.cols = d.k;
    a.k = d.f;
    a.segments = wu ? 2 : 1;
    a.halves = a.parts = 1;
    a.out[0] = gx;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(d0) && aligned_rows(og) && aligned_rows(ou) && whole && whole_h;
    rc = run_rows<true, OUT_PLAIN>(d.dtype, a, g, (int64_t)d.f * og.ld, tile_rows(d, d.k, false), aligned, s);
  }
  if (rc == QCONV_OK && gwg) {
    GemmArgs a = {};
    a.r[0] = d0;
    a.r[1] = d1;
    a.c[0] = ox;
    a.rows = d.f;
    a.cols = d.k;
    a.segments = a.parts = 1;
    a.halves = wu ? 2 : 1;
    a.out[0] = gwg;
    a.out[1] = gwu ? gwu : gwg;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(d0) && aligned_rows(ox) && whole && whole_h;
    const int tile = tile_weights(d, a.halves);
    const int64_t step = (int64_t)d.f * d.k;
    rc = d.dtype == QCONV_F16 ? run_weights_t<F16>(a, g, step, tile, aligned, s)
                              : run_weights_t<BF16>(a, g, step, tile, aligned, s);
  }
  return rc;
}

}  // namespace qc
