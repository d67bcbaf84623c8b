// gradnorm.hip -- the norm over all gradients of a model and clipping by it:
//   norm = sqrt(sum over tensors and values of g^2),
//   out = c g,  c = max_norm / norm where norm > max_norm, else 1.
// Bound by HBM: every gradient is read once for the norm and, where c is not
// already known to leave it alone in place, once more for the product.
// The squares are summed in fp64, whose rate (39 T fma/s) is far above what
// the loads deliver, so no large or small gradient over- or underflows and
// the order of the sum does not show in the fp32 result.
// The tensors' addresses travel in the kernel arguments, so that a call needs
// no copy to the device and can be captured into a graph.
#include "dense.h"

#include "qconv_internal.h"

namespace qc {

namespace {

constexpr int PER_LAUNCH = 112;  // tensors of one launch: the table stays under the 4 KB of kernel arguments
constexpr int CHUNK = 16384;     // values of one piece of work; a multiple of 8, so pieces of a tensor are aligned alike
constexpr int MAX_PARTS = 2048;  // partial sums of a call, if it has at most so many launches

struct Table {
  const void* in[PER_LAUNCH];
  void* out[PER_LAUNCH];
  int64_t numel[PER_LAUNCH];
  int last[PER_LAUNCH];  // chunks up to and with this tensor
  uint8_t type[PER_LAUNCH];
  int count, chunks;
};
static_assert(sizeof(Table) <= 3900, "kernel arguments");

template <int DT>
__device__ __forceinline__ float value_at(const void* p, int64_t i) {
  if constexpr (DT == QCONV_F32) return ((const float*)p)[i];
  if constexpr (DT == QCONV_F16) return F16::up(((const uint16_t*)p)[i]);
  return BF16::up(((const uint16_t*)p)[i]);
}
template <int DT>
__device__ __forceinline__ void put_at(void* p, int64_t i, float v) {
  if constexpr (DT == QCONV_F32) ((float*)p)[i] = v;
  else if constexpr (DT == QCONV_F16) ((uint16_t*)p)[i] = F16::down(v);
  else ((uint16_t*)p)[i] = BF16::down(v);
}

// Tensor of a chunk and the chunk's first value.
__device__ __forceinline__ int find(const Table& t, int chunk, int64_t* start) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (t.last[mid] > chunk) hi = mid;
    else lo = mid + 1;
  }
  *start = (int64_t)(chunk - (lo ? t.last[lo - 1] : 0)) * CHUNK;
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <int DT>
__device__ __forceinline__ double squares(const void* p, int64_t b, int64_t e) {
  double s = 0.0;
  for (int64_t i = b + threadIdx.x; i < e; i += 256) {
    const double v = (double)value_at<DT>(p, i);
    s = fma(v, v, s);
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(Table t, double* parts) {
  __shared__ double lds[4];
  double s = 0.0;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    int64_t b;
    const int i = find(t, c, &b);
    const int64_t e = b + CHUNK < t.numel[i] ? b + CHUNK : t.numel[i];
    if (t.type[i] == QCONV_F32) s += squares<QCONV_F32>(t.in[i], b, e);
    else if (t.type[i] == QCONV_F16) s += squares<QCONV_F16>(t.in[i], b, e);
    else s += squares<QCONV_BF16>(t.in[i], b, e);
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// Every block of a launch adds the same partial sums in the same order.
__device__ __forceinline__ double norm_of(const double* parts, int n, double* lds) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += parts[i];
  return sqrt(block_sum(s, lds));
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* parts, int n, float* norm) {
  __shared__ double lds[4];
  const double v = norm_of(parts, n, lds);
  if (threadIdx.x == 0) *norm = (float)v;
}

template <int DT>
__device__ __forceinline__ void scale(const void* in, void* out, int64_t b, int64_t e, float c) {
  for (int64_t i = b + threadIdx.x; i < e; i += 256) put_at<DT>(out, i, value_at<DT>(in, i) * c);
}

__global__ __launch_bounds__(256) void grad_scale_kernel(Table t, const double* parts, int n, float max_norm,
                                                         float* norm) {
  __shared__ double lds[4];
  const double v = norm_of(parts, n, lds);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  const float c = v > (double)max_norm ? (float)((double)max_norm / v) : 1.0f;
  for (int k = blockIdx.x; k < t.chunks; k += gridDim.x) {
    int64_t b;
    const int i = find(t, k, &b);
    if (c == 1.0f && t.in[i] == t.out[i]) continue;
    const int64_t e = b + CHUNK < t.numel[i] ? b + CHUNK : t.numel[i];
    if (t.type[i] == QCONV_F32) scale<QCONV_F32>(t.in[i], t.out[i], b, e, c);
    else if (t.type[i] == QCONV_F16) scale<QCONV_F16>(t.in[i], t.out[i], b, e, c);
    else scale<QCONV_BF16>(t.in[i], t.out[i], b, e, c);
  }
}

int launches_of(int count) { return ceil_div(count, PER_LAUNCH); }

// Blocks of a squares launch over `chunks` pieces.
int norm_blocks(int launches, int64_t chunks) {
  const int most = MAX_PARTS / launches < 64 ? 64 : MAX_PARTS / launches;
  return (int)(chunks < most ? chunks : most);
}

// Fills the table of launch `l` (the caller bounds numel so that the chunks
// count in an int).
void fill(Table* t, int l, int count, const void* const* grads, void* const* out, const int64_t* numel,
          const int* dtypes) {
  int64_t chunks = 0;
  t->count = 0;
  for (int i = l * PER_LAUNCH; i < count && i < (l + 1) * PER_LAUNCH; ++i) {
    const int k = t->count++;
    chunks += (numel[i] + CHUNK - 1) / CHUNK;
    t->in[k] = grads[i];
    t->out[k] = out ? out[i] : nullptr;
    t->numel[k] = numel[i];
    t->type[k] = (uint8_t)dtypes[i];
    t->last[k] = (int)chunks;
  }
  t->chunks = (int)chunks;
}

// The squares of all tensors; *n = partial sums written.
int run_squares(int count, const void* const* grads, const int64_t* numel, const int* dtypes, double* parts, int* n,
                hipStream_t s) {
  *n = 0;
  const int launches = launches_of(count);
  for (int l = 0; l < launches; ++l) {
    Table t;
    fill(&t, l, count, grads, nullptr, numel, dtypes);
    if (t.chunks == 0) continue;
    const int blocks = norm_blocks(launches, t.chunks);
    grad_squares_kernel<<<blocks, 256, 0, s>>>(t, parts + *n);
    *n += blocks;
    const int rc = hip_status();
    if (rc) return rc;
  }
  return QCONV_OK;
}

}  // namespace

size_t grad_norm_bytes(int count, const int64_t* numel) {
  const int launches = launches_of(count);
  size_t n = 0;
  for (int l = 0; l < launches; ++l) {
    int64_t chunks = 0;
    for (int i = l * PER_LAUNCH; i < count && i < (l + 1) * PER_LAUNCH; ++i) chunks += (numel[i] + CHUNK - 1) / CHUNK;
    n += (size_t)norm_blocks(launches, chunks);
  }
  return n * sizeof(double);
}

int launch_grad_norm(int count, const void* const* grads, const int64_t* numel, const int* dtypes, float* norm,
                     void* ws, hipStream_t s) {
  int n;
  const int rc = run_squares(count, grads, numel, dtypes, (double*)ws, &n, s);
  if (rc) return rc;
  grad_norm_kernel<<<1, 256, 0, s>>>((const double*)ws, n, norm);
  return hip_status();
}

int launch_clip_grads(int count, const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes,
                      float max_norm, float* norm, void* ws, hipStream_t s) {
  int n;
  int rc = run_squares(count, grads, numel, dtypes, (double*)ws, &n, s);
  if (rc) return rc;
  bool told = false;  // the first launch with work writes the norm
  for (int l = 0; l < launches_of(count); ++l) {
    Table t;
    fill(&t, l, count, grads, out, numel, dtypes);
    if (t.chunks == 0) continue;
    const int blocks = t.chunks < 2048 ? t.chunks : 2048;
    grad_scale_kernel<<<blocks, 256, 0, s>>>(t, (const double*)ws, n, max_norm, told ? nullptr : norm);
    told = true;
    if ((rc = hip_status())) return rc;
  }
  if (!told) grad_norm_kernel<<<1, 256, 0, s>>>((const double*)ws, 0, norm);
  return hip_status();
}

}  // namespace qc
