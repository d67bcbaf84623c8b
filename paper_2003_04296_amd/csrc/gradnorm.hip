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

// Values of a type in 16 bytes, their widening and their rounding.
template <int DT>
struct Values {
  static constexpr int N = DT == QCONV_F32 ? 4 : 8, SIZE = DT == QCONV_F32 ? 4 : 2;
  __device__ __forceinline__ static float one(const char* p, int64_t i) {
    if constexpr (DT == QCONV_F32) return ((const float*)p)[i];
    if constexpr (DT == QCONV_F16) return F16::up(((const uint16_t*)p)[i]);
    return BF16::up(((const uint16_t*)p)[i]);
  }
  __device__ __forceinline__ static void put(char* p, int64_t i, float v) {
    if constexpr (DT == QCONV_F32) ((float*)p)[i] = v;
    else if constexpr (DT == QCONV_F16) ((uint16_t*)p)[i] = F16::down(v);
    else ((uint16_t*)p)[i] = BF16::down(v);
  }
  __device__ __forceinline__ static void widen(v4u w, float v[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (DT == QCONV_F32) v[e] = __uint_as_float(w[e]);
      else if constexpr (DT == QCONV_F16) v[e] = F16::up((uint16_t)(w[e / 2] >> (16 * (e & 1))));
      else v[e] = BF16::up((uint16_t)(w[e / 2] >> (16 * (e & 1))));
    }
  }
  __device__ __forceinline__ static v4u narrow(const float v[N]) {
    v4u w = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (DT == QCONV_F32) w[e] = __float_as_uint(v[e]);
      else if constexpr (DT == QCONV_F16) w[e / 2] |= (uint32_t)F16::down(v[e]) << (16 * (e & 1));
      else w[e / 2] |= (uint32_t)BF16::down(v[e]) << (16 * (e & 1));
    }
    return w;
  }
};

// The values [b, e) of a tensor at p in three parts: up to 16-byte alignment,
// whole 16-byte groups, and the rest.
struct Parts {
  int64_t first, groups, rest;  // first value of the groups, their number, first value after them
};
template <int DT>
__device__ __forceinline__ Parts parts_of(const void* p, int64_t b, int64_t e) {
  typedef Values<DT> V;
  const int64_t skew = (int64_t)((uintptr_t)p / V::SIZE + b) & (V::N - 1);
  Parts r;
  r.first = b + (skew ? V::N - skew : 0);
  if (r.first > e) r.first = e;
  r.groups = (e - r.first) / V::N;
  r.rest = r.first + r.groups * V::N;
  return r;
}

// A walk over the chunks [from, to) of a launch; blocks take neighbouring
// runs, so that the tensor of a chunk is found once and then followed.
struct Run {
  int from, to;
};
__device__ __forceinline__ Run run_of(const Table& t) {
  return {(int)((int64_t)t.chunks * blockIdx.x / gridDim.x), (int)((int64_t)t.chunks * (blockIdx.x + 1) / gridDim.x)};
}
__device__ __forceinline__ int tensor_of(const Table& t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (t.last[mid] > chunk) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
// The first value of a chunk of tensor i, and the one after its last.
__device__ __forceinline__ void range_of(const Table& t, int i, int chunk, int64_t* b, int64_t* e) {
  *b = (int64_t)(chunk - (i ? t.last[i - 1] : 0)) * CHUNK;
  *e = *b + CHUNK < t.numel[i] ? *b + CHUNK : t.numel[i];
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Groups loaded by a thread before any is used: the loads of a wave have to
// cover the memory's latency.
constexpr int AHEAD = 8;

template <int DT>
__device__ __forceinline__ double squares(const void* p, int64_t b, int64_t e) {
  typedef Values<DT> V;
  const Parts r = parts_of<DT>(p, b, e);
  const v4u* g = (const v4u*)((const char*)p + r.first * V::SIZE);
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < r.groups; i += 256 * AHEAD) {
    v4u w[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) w[j] = i + j * 256 < r.groups ? g[i + j * 256] : v4u{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      float v[V::N];
      V::widen(w[j], v);
#pragma unroll
      for (int k = 0; k < V::N; ++k) s = fma((double)v[k], (double)v[k], s);
    }
  }
  const int64_t head = b + threadIdx.x, tail = r.rest + threadIdx.x;  // at most 7 values each
  if (head < r.first) {
    const double v = (double)V::one((const char*)p, head);
    s = fma(v, v, s);
  }
  if (tail < e) {
    const double v = (double)V::one((const char*)p, tail);
    s = fma(v, v, s);
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(Table t, double* parts) {
  __shared__ double lds[4];
  const Run run = run_of(t);
  double s = 0.0;
  int i = tensor_of(t, run.from);
  for (int c = run.from; c < run.to; ++c) {
    while (c >= t.last[i]) ++i;
    int64_t b, e;
    range_of(t, i, c, &b, &e);
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

// Sixteen bytes from any address a value may have.
template <int DT>
__device__ __forceinline__ v4u load16(const char* p) {
  struct __attribute__((packed, aligned(Values<DT>::SIZE))) U {
    v4u v;
  };
  return reinterpret_cast<const U*>(p)->v;
}

// Stores are aligned; loads need not be, where the two tensors start differently.
template <int DT>
__device__ __forceinline__ void scale(const void* in, void* out, int64_t b, int64_t e, float c) {
  typedef Values<DT> V;
  const Parts r = parts_of<DT>(out, b, e);
  const char* g = (const char*)in + r.first * V::SIZE;
  v4u* o = (v4u*)((char*)out + r.first * V::SIZE);
  for (int64_t i = threadIdx.x; i < r.groups; i += 256 * AHEAD) {
    v4u w[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      w[j] = i + j * 256 < r.groups ? load16<DT>(g + (i + j * 256) * 16) : v4u{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      float v[V::N];
      V::widen(w[j], v);
#pragma unroll
      for (int k = 0; k < V::N; ++k) v[k] *= c;
      if (i + j * 256 < r.groups) __builtin_nontemporal_store(V::narrow(v), o + i + j * 256);
    }
  }
  const int64_t head = b + threadIdx.x, tail = r.rest + threadIdx.x;
  if (head < r.first) V::put((char*)out, head, V::one((const char*)in, head) * c);
  if (tail < e) V::put((char*)out, tail, V::one((const char*)in, tail) * c);
}

// Each block walks its run backwards: what the norm's pass read last is what
// the 256 MB cache still holds.
__global__ __launch_bounds__(256) void grad_scale_kernel(Table t, const double* parts, int n, float max_norm,
                                                         float* norm) {
  __shared__ double lds[4];
  const double v = norm_of(parts, n, lds);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  const float c = v > (double)max_norm ? (float)((double)max_norm / v) : 1.0f;
  const Run run = run_of(t);
  int i = tensor_of(t, run.to - 1);
  for (int k = run.to - 1; k >= run.from; --k) {
    while (i > 0 && k < t.last[i - 1]) --i;
    if (c == 1.0f && t.in[i] == t.out[i]) continue;
    int64_t b, e;
    range_of(t, i, k, &b, &e);
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
