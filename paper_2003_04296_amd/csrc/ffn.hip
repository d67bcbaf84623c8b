// ffn.hip -- the gated feed-forward block in 16-bit types, forward and
// backward, as three matrix products on the matrix cores:
//   forward   g = x Wg^T, u = x Wu^T, h = act(g) u      (one launch)
//   gradients dg = gh u act'(g), du = gh act(g)         (elementwise)
//             gx = dg Wg + du Wu;  gWg = dg^T x, gWu = du^T x
// The kernels are those of dense_gemm.h; few tokens go forward through
// dense_rows.h, which reads the weights once without tiles of x.
#include "dense_gemm.h"
#include "dense_rows.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// dg and du of four hidden features per thread, into [m][2][fp] with the
// columns past f zero (gx's products run over all fp of them).  They are
// rounded to the tensors' type, once, because the matrix cores take 16-bit
// operands; g and u themselves stay in fp32 between the passes.  The gradients'
// error is 1.4 times that of fp32 factors (two roundings in place of one), and a
// factor past fp16's 65504 is infinite, as a gradient of that type is.  Two parts
// per factor would hold both and double the backward's products.  Bound by HBM:
// 8192 tokens of 16384 features read 1.3 GB and write 0.5 in 352 us, 5.3 TB/s.
template <class T, int ACT>
__global__ __launch_bounds__(256) void ffn_slopes_kernel(const float* __restrict__ pre, const uint16_t* __restrict__ gh,
                                                         int64_t ld_h, int m, int f, int fp,
                                                         uint16_t* __restrict__ d) {
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

// The products of two 16-bit operands in the given forms.
template <class T, bool RCOL, bool CCOL, int OUT>
int run_gemm_t(GemmArgs& a, const GemmPlan& p, bool aligned, hipStream_t s) {
  constexpr bool PAIR = OUT == OUT_GATED;
  constexpr int KS = RCOL || CCOL ? 32 : 64;
  a.parts = p.parts;
  if (!aligned)
    return run_gemm_tiles<T, Stage16<KS, 128, 256, 0, RCOL, false, false>, Stage16<KS, 128, 256, 1, CCOL, false, PAIR>,
                          OUT, 128>(a, s);
  if (p.tile == 256)
    return run_gemm_tiles<T, Stage16<KS, 256, 512, 0, RCOL, true, false>, Stage16<KS, 256, 512, 1, CCOL, true, PAIR>,
                          OUT, 256>(a, s);
  return run_gemm_tiles<T, Stage16<KS, 128, 256, 0, RCOL, true, false>, Stage16<KS, 128, 256, 1, CCOL, true, PAIR>,
                        OUT, 128>(a, s);
}

template <bool RCOL, bool CCOL, int OUT>
int run_gemm(int dtype, GemmArgs& a, const GemmPlan& p, bool aligned, hipStream_t s) {
  return dtype == QCONV_F16 ? run_gemm_t<F16, RCOL, CCOL, OUT>(a, p, aligned, s)
                            : run_gemm_t<BF16, RCOL, CCOL, OUT>(a, p, aligned, s);
}

// Products of the forward, of gx and of the weight gradients.
GemmPlan plan_h(const qconv_ffn_desc& d, bool aligned) {
  return gemm_plan(d.m, d.f, d.k, 1, true, aligned, false);
}
GemmPlan plan_gx(const qconv_ffn_desc& d, bool aligned) {
  return gemm_plan(d.m, d.k, 2 * (int64_t)d.f, 1, false, aligned, true);
}
GemmPlan plan_gw(const qconv_ffn_desc& d, bool aligned) {
  return gemm_plan(d.f, d.k, d.m, 2, false, aligned, false);
}

template <class T>
int run_slopes(const qconv_ffn_desc& d, const float* pre, const void* gh, int fp, uint16_t* out, hipStream_t s) {
  const int64_t n = (int64_t)d.m * (fp / 4);
  const unsigned grid = (unsigned)(n < (1 << 23) ? (n + 255) / 256 : 1 << 15);
  const uint16_t* g = (const uint16_t*)gh;
  if (d.act == QCONV_ACT_SILU)
    ffn_slopes_kernel<T, QCONV_ACT_SILU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  else if (d.act == QCONV_ACT_GELU)
    ffn_slopes_kernel<T, QCONV_ACT_GELU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  else
    ffn_slopes_kernel<T, QCONV_ACT_RELU><<<grid, 256, 0, s>>>(pre, g, d.ld_h, d.m, d.f, fp, out);
  return hip_status();
}

}  // namespace

// Copies of x and the weights in aligned rows, first in the workspace.  The
// forward makes them from as many tokens on as make up for copying both weights
// where these are large; us with copies and without:
//   4095 -> 16384  238 and 114 at 100 tokens, 261 and 220 at 384, 351 and 441 at 800
//   2047 -> 4001   36 and 36, 50 and 55, 61 and 78
//   1001 -> 1000   25 and 32, 26 and 30, 26 and 37
// The backward, which reads the weights down their columns, always does:
//   4095 -> 8192   237 and 371 for one token, 296 and 621 for 200
//   1001 -> 1000   33 and 62, 42 and 73
constexpr int COPY_LEAST = 384;
static size_t copies_bytes(const qconv_ffn_desc& d, bool forward) {
  if (forward && d.m < COPY_LEAST) return 0;
  return realigns(d.k, d.ld_x, d.ld_w) ? realign_bytes(d.m, d.k) + 2 * realign_bytes(d.f, d.k) : 0;
}

size_t ffn_forward_bytes(const qconv_ffn_desc& d) {
  if (d.m <= ROWS_MOST) return 0;
  const size_t p = plan_h(d, false).bytes, q = plan_h(d, true).bytes;
  return copies_bytes(d, true) + (p > q ? p : q);
}

int launch_ffn_forward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, void* h, float* pre,
                       void* ws, hipStream_t s) {
  if (d.m == 0) return QCONV_OK;
  if (d.m <= ROWS_MOST) {
    RowsArgs r = {};
    r.x = (const uint16_t*)x;
    r.ld_x = d.ld_x;
    r.ld_w = d.ld_w;
    r.ld_y = d.ld_h;
    r.w[0] = wg;
    r.w[1] = wu;
    r.y = (uint16_t*)h;
    r.pre = pre;
    r.ld_pre = (int)round_up(d.f, 8);
    r.m = d.m;
    r.n = d.f;
    r.k = d.k;
    r.act = d.act;
    if (d.m <= FEW_MOST) return d.dtype == QCONV_F16 ? run_dense_few<F16, 0, 2>(r, s) : run_dense_few<BF16, 0, 2>(r, s);
    return d.dtype == QCONV_F16 ? run_dense_rows<F16, Dense16, 2>(r, s) : run_dense_rows<BF16, Dense16, 2>(r, s);
  }
  GemmArgs a = {};
  a.r[0] = {(const uint16_t*)x, d.ld_x};
  a.c[0] = {(const uint16_t*)wg, d.ld_w};
  a.c[1] = {(const uint16_t*)wu, d.ld_w};
  a.rows = d.m;
  a.cols = d.f;
  a.k = d.k;
  a.segments = a.halves = 1;
  a.out[0] = h;
  a.ld_out = d.ld_h;
  a.pre = pre;
  a.ld_pre = (int)round_up(d.f, 8);
  a.act = d.act;
  if (copies_bytes(d, true)) {
    Realigner re(d.k, ws);
    re.add(a.r[0], d.m);
    re.add_pair(a.c[0], a.c[1], d.f);
    const int rc = re.run(s);
    if (rc) return rc;
    a.k = re.a.kp;
  }
  const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && aligned_rows(a.c[1]) && a.k % 8 == 0;
  a.part = (float*)((char*)ws + copies_bytes(d, true));
  return run_gemm<false, false, OUT_GATED>(d.dtype, a, plan_h(d, aligned), aligned, s);
}

// The copies, dg and du, then the parts of whichever product has more of them.
static size_t slopes_bytes(const qconv_ffn_desc& d) { return (size_t)round_up((int64_t)d.m * 2 * round_up(d.f, 8) * 2, 16); }
size_t ffn_backward_bytes(const qconv_ffn_desc& d) {
  size_t most = 0;
  for (bool aligned : {false, true})
    for (const GemmPlan& p : {plan_gx(d, aligned), plan_gw(d, aligned)})
      if (p.bytes > most) most = p.bytes;
  return copies_bytes(d, false) + slopes_bytes(d) + most;
}

int launch_ffn_backward(const qconv_ffn_desc& d, const void* x, const void* wg, const void* wu, const float* pre,
                        const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s) {
  const int fp = (int)round_up(d.f, 8);
  uint16_t* dgu = (uint16_t*)((char*)ws + copies_bytes(d, false));
  float* part = (float*)((char*)dgu + slopes_bytes(d));
  int rc = QCONV_OK;
  Operand ox = {(const uint16_t*)x, d.ld_x}, og = {(const uint16_t*)wg, d.ld_w}, ou = {(const uint16_t*)wu, d.ld_w};
  bool whole = d.k % 8 == 0;  // rows end with 16 bytes
  if (copies_bytes(d, false)) {
    Realigner re(d.k, ws);
    if (gwg) re.add(ox, d.m);
    if (gx && d.m > 0) re.add_pair(og, ou, d.f);
    rc = re.run(s);
    if (rc) return rc;
    whole = true;
  }
  if (d.m > 0)
    rc = d.dtype == QCONV_F16 ? run_slopes<F16>(d, pre, gh, fp, dgu, s) : run_slopes<BF16>(d, pre, gh, fp, dgu, s);
  if (rc == QCONV_OK && gx && d.m > 0) {
    GemmArgs a = {};
    a.r[0] = {dgu, 2 * (int64_t)fp};
    a.r[1] = {dgu + fp, 2 * (int64_t)fp};
    a.c[0] = og;
    a.c[1] = ou;
    a.rows = d.m;
    a.cols = d.k;
    a.k = d.f;
    a.segments = 2;
    a.halves = 1;
    a.out[0] = gx;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && aligned_rows(a.c[1]) && whole;
    a.part = part;
    rc = run_gemm<false, true, OUT_PLAIN>(d.dtype, a, plan_gx(d, aligned), aligned, s);
  }
  if (rc == QCONV_OK && gwg) {
    GemmArgs a = {};
    a.r[0] = {dgu, 2 * (int64_t)fp};
    a.r[1] = {dgu + fp, 2 * (int64_t)fp};
    a.c[0] = ox;
    a.rows = d.f;
    a.cols = d.k;
    a.k = d.m;
    a.segments = 1;
    a.halves = 2;
    a.out[0] = gwg;
    a.out[1] = gwu;
    a.ld_out = d.k;
    const bool aligned = aligned_rows(a.r[0]) && aligned_rows(a.c[0]) && whole;
    a.part = part;
    rc = run_gemm<true, true, OUT_PLAIN>(d.dtype, a, plan_gw(d, aligned), aligned, s);
  }
  return rc;
}

}  // namespace qc
