// moe_rows.hip -- rows of a batch that go to different weights: the order that
// brings each expert's rows together, rows copied into it and back, and their
// gradients.
//   sort     key(i) = id i where 0 <= id < groups, else groups; order = the
//            stable permutation by key, place = its inverse, offsets[g] = how
//            many keys are below g
//   gather   xs[place[t, s]] = x[t]
//   combine  y[t] = sum_s w[t, s] ys[place[t, s]]
//   back     gys[place[t, s]] = w[t, s] gy[t],  gw[t, s] = <gy[t], ys[place[t, s]]>
#include "dense.h"
#include "moe.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// ---------------------------------------------------------------------------
// The order
// ---------------------------------------------------------------------------

struct SortArgs {
  const void* ids;
  int wide;  // 64-bit ids
  int slots;
  int64_t ld;
  int n, groups;
  int chunk;        // ids per block
  int* hist;        // [groups + 1][blocks]: ids of each key in each block
  int *offsets, *order, *place;
};

// Id i as a key.
__device__ __forceinline__ int sort_key(const SortArgs& a, int i) {
  const int64_t at = a.ld == a.slots ? i : (int64_t)(i / a.slots) * a.ld + i % a.slots;
  const int64_t id = a.wide ? ((const int64_t*)a.ids)[at] : ((const int*)a.ids)[at];
  return id >= 0 && id < a.groups ? (int)id : a.groups;
}

// The lanes of `on` that hold this lane's key.
__device__ __forceinline__ uint64_t same_key(int key, int bits, uint64_t on) {
  uint64_t m = on;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(key >> b & 1);
    m &= key >> b & 1 ? set : ~set;
  }
  return m;
}

// Exclusive prefix sums of v[0, n) by a block of NT threads, in place; the sum
// of all in every thread.  tmp: a word per wave.
template <int NT>
__device__ __forceinline__ int block_scan(int* v, int n, int* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (n + NT - 1) / NT, b = (int)threadIdx.x * per < n ? (int)threadIdx.x * per : n, e = b + per < n ? b + per : n;
  int mine = 0;
  for (int i = b; i < e; ++i) mine += v[i];
  int incl = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) tmp[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int s = tmp[w];
    before += w < wave ? s : 0;
    all += s;
  }
  int at = before + incl - mine;
  for (int i = b; i < e; ++i) {
    const int s = v[i];
    v[i] = at;
    at += s;
  }
  __syncthreads();
  return all;
}

// Counts of each key in a block's ids.
__global__ __launch_bounds__(1024) void moe_count_kernel(SortArgs a) {
  __shared__ int cnt[MOE_GROUPS_MOST + 1];
  for (int g = threadIdx.x; g <= a.groups; g += 1024) cnt[g] = 0;
  __syncthreads();
  const int64_t b = (int64_t)blockIdx.x * a.chunk, e = b + a.chunk < a.n ? b + a.chunk : a.n;
  for (int64_t i = b + threadIdx.x; i < e; i += 1024) atomicAdd(&cnt[sort_key(a, (int)i)], 1);
  __syncthreads();
  for (int g = threadIdx.x; g <= a.groups; g += 1024) a.hist[(int64_t)g * gridDim.x + blockIdx.x] = cnt[g];
}

// Ranks a block's ids and writes order, place and (the first block) offsets.
// Each wave owns a run of the ids and counts of its own in LDS, so that ranks
// follow the ids' order whatever the waves' timing: the sums over earlier blocks
// (from their counts, which every block reads: at most 2^17 words, a key's in a
// row), earlier
// waves and smaller keys are the start of a wave's rows of a key.
// Bound by latency (32768 x 8 ids move 4 MB): 128 blocks of 2048 ids 8.8 us, of which
// the counts of all blocks took 20 more while one thread summed each key, one block of
// 64 ids 3.4.
template <int NW, int BUCKETS>
__global__ __launch_bounds__(NW * 64) void moe_rank_kernel(SortArgs a) {
  constexpr int NT = NW * 64;
  __shared__ int cnt[NW][BUCKETS];
  __shared__ int base[BUCKETS], start[BUCKETS];
  __shared__ int tmp[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int buckets = a.groups + 1, bits = 32 - __clz(a.groups);
  for (int w = 0; w < NW; ++w)
    for (int g = threadIdx.x; g < buckets; g += NT) cnt[w][g] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.chunk;
  const int here = (int)(first + a.chunk < a.n ? a.chunk : a.n - first);
  const int run = (ceil_div(here, NW) + 63) & ~63;
  const int b = wave * run < here ? wave * run : here, e = b + run < here ? b + run : here;
  for (int i = b + lane; i < e; i += 64) atomicAdd(&cnt[wave][sort_key(a, (int)first + i)], 1);
  __syncthreads();
  // per key: in base all its rows, in start those of earlier blocks.  Eight lanes
  // sum the blocks' counts of one key.
  if (a.hist) {
    const int blocks = gridDim.x;
    const int in = lane & 7;
    for (int g0 = wave * 8; g0 < buckets; g0 += NT / 8) {
      const int g = g0 + lane / 8;
      const int* h = a.hist + (int64_t)(g < buckets ? g : 0) * blocks;
      int before = 0, total = 0;
      for (int k0 = 0; k0 < blocks; k0 += 64) {
        int c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = k0 + i * 8 + in < blocks ? h[k0 + i * 8 + in] : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          before += k0 + i * 8 + in < (int)blockIdx.x ? c[i] : 0;
          total += c[i];
        }
      }
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) {
        before += __shfl_xor(before, d);
        total += __shfl_xor(total, d);
      }
      if (in == 0 && g < buckets) {
        base[g] = total;
        start[g] = before;
      }
    }
  } else {
    for (int g = threadIdx.x; g < buckets; g += NT) {
      int total = 0;
      for (int w = 0; w < NW; ++w) total += cnt[w][g];
      base[g] = total;
      start[g] = 0;
    }
  }
  __syncthreads();
  block_scan<NT>(base, buckets, tmp);
  for (int g = threadIdx.x; g < buckets; g += NT) {
    int at = base[g] + start[g];
    for (int w = 0; w < NW; ++w) {
      const int c = cnt[w][g];
      cnt[w][g] = at;
      at += c;
    }
  }
  if (blockIdx.x == 0)
    for (int g = threadIdx.x; g < buckets; g += NT) a.offsets[g] = base[g];
  __syncthreads();
  for (int i = b; i < e; i += 64) {
    const bool in = i + lane < e;
    const int at = (int)first + i + lane, key = in ? sort_key(a, at) : 0;
    const uint64_t mine = same_key(key, bits, __ballot(in));
    const int before = __popcll(mine & ((1ull << lane) - 1));
    const int r = cnt[wave][key] + before;
    // the wave's lanes have read before the first of each key writes
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in) {
      if (before == 0) cnt[wave][key] = r + __popcll(mine);
      a.order[r] = at;
      a.place[at] = key < a.groups ? r : -1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Up to SORT_ONE ids are one block's, in one launch; more are taken SORT_CHUNK a block.
// us in one block and in several (in a graph): 8 groups 6.5 and 7.8 at 4096 ids, 9.6
// and 7.9 at 8192; 1000 groups 9.2 and 13.9, 14.0 and 14.3.  With 1024, 2048 and 4096
// ids a block: 8.5, 9.5 and 11.9 at 32768 ids, 13.2, 11.9 and 12.9 at 262144.
constexpr int SORT_ONE = 4096;
constexpr int SORT_CHUNK = 2048;

int sort_blocks(int n, int groups) {
  if (n <= SORT_ONE) return 1;
  const int most = (1 << 17) / (groups + 1) < 256 ? (1 << 17) / (groups + 1) : 256;
  const int want = ceil_div(n, SORT_CHUNK);
  return want < most ? want : most;
}

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------

// Values of a type in 16 bytes.  Rows may start at any address that a value may
// have: global loads and stores of 16 bytes take them.
struct F32 {
  static constexpr int N = 4;
  typedef float E;
  struct __attribute__((packed, aligned(4))) Any {
    v4u v;
  };
  __device__ __forceinline__ static float up(float v) { return v; }
  __device__ __forceinline__ static float down(float v) { return v; }
  __device__ __forceinline__ static void widen(v4u w, float v[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = __uint_as_float(w[e]);
  }
  __device__ __forceinline__ static v4u narrow(const float v[N]) {
    return v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <class T>
struct Half {
  static constexpr int N = 8;
  typedef uint16_t E;
  typedef U128 Any;
  __device__ __forceinline__ static float up(uint16_t v) { return T::up(v); }
  __device__ __forceinline__ static uint16_t down(float v) { return T::down(v); }
  __device__ __forceinline__ static void widen(v4u w, float v[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = T::up((uint16_t)(w[e / 2] >> (16 * (e & 1))));
  }
  __device__ __forceinline__ static v4u narrow(const float v[N]) {
    v4u w;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = T::down(v[2 * e]) | (uint32_t)T::down(v[2 * e + 1]) << 16;
    return w;
  }
};

// The values [c, c + N) of a row of `width`; what lies past it is 0 and not read,
// and not written.
template <class V>
__device__ __forceinline__ v4u load_part(const typename V::E* row, int c, int width) {
  if (c + V::N <= width) return reinterpret_cast<const typename V::Any*>(row + c)->v;
  typename V::E t[V::N];
#pragma unroll
  for (int e = 0; e < V::N; ++e) t[e] = c + e < width ? row[c + e] : (typename V::E)0;
  return __builtin_bit_cast(v4u, t);
}
template <class V>
__device__ __forceinline__ void store_part(typename V::E* row, int c, int width, v4u v) {
  if (c + V::N <= width) {
    reinterpret_cast<typename V::Any*>(row + c)->v = v;
    return;
  }
  typename V::E t[V::N];
  __builtin_memcpy(t, &v, 16);
#pragma unroll
  for (int e = 0; e < V::N; ++e)
    if (c + e < width) row[c + e] = t[e];
}

struct RowArgs {
  const void *x, *gy;       // rows of tokens (gather, the gradient of combine)
  const void* ys;           // rows of experts (combine and its gradient)
  void *y, *rows;           // of tokens; of experts
  const float* weights;     // [tokens][slots] or NULL: 1
  float* gw;
  const int* place;         // [tokens][slots]
  int64_t ld_t, ld_e;       // row strides: tokens' operand, experts' rows
  int64_t ld_o;             // of a token's result
  int64_t n;                // tokens * slots
  int tokens, slots, width;
  int per;                  // 16-byte parts of a row
  int lanes, segments;      // lanes that share a row, and pieces of `lanes` parts it takes
};

// A group of `lanes` lanes takes `lanes` parts of one token's row: the item.
// f(token, first value of this lane's part), for the lanes that have one.
template <int N, class F>
__device__ __forceinline__ void each_part(const RowArgs& a, F&& f) {
  const int lane = threadIdx.x & (a.lanes - 1);
  const uint32_t items = (uint32_t)a.tokens * a.segments, step = gridDim.x * (256u / a.lanes);
  for (uint32_t i = blockIdx.x * (256u / a.lanes) + threadIdx.x / a.lanes; i < items; i += step) {
    const uint32_t t = a.segments == 1 ? i : i / a.segments;
    const int p = (int)(i - t * a.segments) * a.lanes + lane;
    if (p < a.per) f((int)t, p * N);
  }
}

// Bound by HBM: a token's row is read once and written once per slot (8192 tokens x 4
// of 4096 bf16: 336 MB in 53 us, 6.3 TB/s).
template <class V>
__global__ __launch_bounds__(256) void moe_gather_kernel(RowArgs a) {
  typedef typename V::E E;
  each_part<V::N>(a, [&](int t, int c) {
    const v4u v = load_part<V>((const E*)a.x + t * a.ld_t, c, a.width);
    for (int s = 0; s < a.slots; ++s) {
      const int64_t r = a.place[(int64_t)t * a.slots + s];
      if (r >= 0 && r < a.n) store_part<V>((E*)a.rows + r * a.ld_e, c, a.width, v);
    }
  });
}

// The sum over a token's slots in fp32, in their order, rounded once.  Four rows
// are loaded at a time.  Bound by HBM: 8192 tokens x 4 of 4096 bf16, 336 MB in 64 us
// from the cache, 80 from memory (4.2 TB/s).
template <class V>
__global__ __launch_bounds__(256) void moe_combine_kernel(RowArgs a) {
  typedef typename V::E E;
  each_part<V::N>(a, [&](int t, int c) {
    float sum[V::N];
#pragma unroll
    for (int e = 0; e < V::N; ++e) sum[e] = 0.0f;
    for (int s0 = 0; s0 < a.slots; s0 += 4) {
      v4u v[4];
      float w[4];
      bool on[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t at = (int64_t)t * a.slots + s0 + i;
        const int64_t r = s0 + i < a.slots ? a.place[at] : -1;
        on[i] = r >= 0 && r < a.n;
        v[i] = on[i] ? load_part<V>((const E*)a.ys + r * a.ld_e, c, a.width) : v4u{0, 0, 0, 0};
        w[i] = on[i] && a.weights ? a.weights[at] : 1.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (on[i]) {
          float f[V::N];
          V::widen(v[i], f);
#pragma unroll
          for (int e = 0; e < V::N; ++e) sum[e] = fmaf(w[i], f[e], sum[e]);
        }
    }
    store_part<V>((E*)a.y + t * a.ld_o, c, a.width, V::narrow(sum));
  });
}

// LANES of a block's 256 threads share a token, four of its slots at a time.  gw is summed per lane, then over the lanes in a fixed
// order.  Bound by HBM: gy and the experts' rows in, the rows' gradients out (8192
// tokens x 4 of 4096 bf16: 604 MB in 103 us, 5.9 TB/s).
template <class V, int LANES>
__global__ __launch_bounds__(256) void moe_combine_back_kernel(RowArgs a) {
  typedef typename V::E E;
  constexpr int PER = 256 / LANES;
  __shared__ float part[LANES > 64 ? 4 : 1][4];
  const int lane = threadIdx.x & (LANES - 1);
  for (int64_t t0 = (int64_t)blockIdx.x * PER; t0 < a.tokens; t0 += (int64_t)gridDim.x * PER) {
    const int64_t t = t0 + threadIdx.x / LANES;
    for (int s0 = 0; s0 < a.slots; s0 += 4) {
      float dot[4], w[4];
      int64_t r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t at = t * a.slots + s0 + i;
        r[i] = t < a.tokens && s0 + i < a.slots ? a.place[at] : -1;
        if (r[i] >= a.n) r[i] = -1;
        w[i] = r[i] >= 0 && a.weights ? a.weights[at] : 1.0f;
        dot[i] = 0.0f;
      }
      if (t < a.tokens)
        for (int p = lane; p < a.per; p += LANES) {
          const int c = p * V::N;
          v4u y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y[i] = r[i] >= 0 && a.gw ? load_part<V>((const E*)a.ys + r[i] * a.ld_e, c, a.width) : v4u{0, 0, 0, 0};
          float g[V::N];
          V::widen(load_part<V>((const E*)a.gy + t * a.ld_t, c, a.width), g);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (r[i] >= 0) {
              float f[V::N];
              if (a.gw) {
                V::widen(y[i], f);
#pragma unroll
                for (int e = 0; e < V::N; ++e) dot[i] = fmaf(g[e], f[e], dot[i]);
              }
              if (a.rows) {
#pragma unroll
                for (int e = 0; e < V::N; ++e) f[e] = w[i] * g[e];
                store_part<V>((E*)a.rows + r[i] * a.ld_o, c, a.width, V::narrow(f));
              }
            }
        }
      if (!a.gw) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d <<= 1) dot[i] += __shfl_xor(dot[i], d);
      if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
          for (int i = 0; i < 4; ++i) part[threadIdx.x >> 6][i] = dot[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) dot[i] = part[0][i] + part[1][i] + part[2][i] + part[3][i];
        __syncthreads();
      }
      if (lane == 0 && t < a.tokens)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (s0 + i < a.slots) a.gw[t * a.slots + s0 + i] = dot[i];
    }
  }
}

// f with the type's values.
template <class F>
int with_values(int dtype, F&& f) {
  if (dtype == QCONV_F32) f(F32{});
  else if (dtype == QCONV_F16) f(Half<F16>{});
  else f(Half<BF16>{});
  return hip_status();
}

RowArgs row_args(const qconv_moe_rows_desc& d, const int* place) {
  RowArgs a = {};
  a.place = place;
  a.tokens = d.tokens;
  a.slots = d.slots;
  a.width = d.width;
  a.n = (int64_t)d.tokens * d.slots;
  a.per = ceil_div(d.width, d.dtype == QCONV_F32 ? 4 : 8);
  a.lanes = 8;
  while (a.lanes < 64 && a.lanes < a.per) a.lanes *= 2;
  a.segments = ceil_div(a.per, a.lanes);
  return a;
}

unsigned row_grid(const RowArgs& a) {
  const int64_t blocks = ((int64_t)a.tokens * a.segments + 256 / a.lanes - 1) / (256 / a.lanes);
  return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
}

}  // namespace

size_t moe_sort_bytes(int n, int groups) {
  const int b = sort_blocks(n, groups);
  return b > 1 ? (size_t)b * (groups + 1) * 4 : 0;
}

int launch_moe_sort(const void* ids, int wide, int tokens, int slots, int64_t ld, int groups, int* offsets, int* order,
                    int* place, void* ws, hipStream_t s) {
  SortArgs a = {};
  a.ids = ids;
  a.wide = wide;
  a.slots = slots;
  a.ld = ld;
  a.n = tokens * slots;
  a.groups = groups;
  a.offsets = offsets;
  a.order = order;
  a.place = place;
  const int blocks = sort_blocks(a.n, groups);
  a.chunk = blocks > 1 ? ceil_div(a.n, blocks) : a.n;
  if (blocks > 1) {
    a.hist = (int*)ws;
    moe_count_kernel<<<blocks, 1024, 0, s>>>(a);
  }
  if (groups < 256)
    moe_rank_kernel<16, 256><<<blocks, 1024, 0, s>>>(a);
  else if (groups < 1024)
    moe_rank_kernel<16, 1024><<<blocks, 1024, 0, s>>>(a);
  else
    moe_rank_kernel<4, MOE_GROUPS_MOST + 1><<<blocks, 256, 0, s>>>(a);
  return hip_status();
}

int launch_moe_gather(const qconv_moe_rows_desc& d, const void* x, const int* place, void* rows, hipStream_t s) {
  if (d.tokens == 0) return QCONV_OK;
  RowArgs a = row_args(d, place);
  a.x = x;
  a.rows = rows;
  a.ld_t = d.ld_tokens;
  a.ld_e = d.ld_rows;
  return with_values(d.dtype, [&](auto v) { moe_gather_kernel<decltype(v)><<<row_grid(a), 256, 0, s>>>(a); });
}

int launch_moe_combine(const qconv_moe_rows_desc& d, const void* ys, const int* place, const float* weights, void* y,
                       hipStream_t s) {
  if (d.tokens == 0) return QCONV_OK;
  RowArgs a = row_args(d, place);
  a.ys = ys;
  a.y = y;
  a.weights = weights;
  a.ld_e = d.ld_rows;
  a.ld_o = d.ld_tokens;
  return with_values(d.dtype, [&](auto v) { moe_combine_kernel<decltype(v)><<<row_grid(a), 256, 0, s>>>(a); });
}

int launch_moe_combine_back(const qconv_moe_rows_desc& d, const void* gy, const void* ys, const int* place,
                            const float* weights, void* gys, int64_t ld_gys, float* gw, hipStream_t s) {
  if (d.tokens == 0 || (!gys && !gw)) return QCONV_OK;
  RowArgs a = row_args(d, place);
  a.gy = gy;
  a.ys = ys;
  a.weights = weights;
  a.rows = gys;
  a.gw = gw;
  a.ld_t = d.ld_tokens;
  a.ld_e = d.ld_rows;
  a.ld_o = ld_gys;
  return with_values(d.dtype, [&](auto v) {
    typedef decltype(v) V;
    auto grid = [&](int lanes) {
      const int64_t b = (a.tokens + 256 / lanes - 1) / (256 / lanes);
      return (unsigned)(b < (1 << 20) ? b : 1 << 20);
    };
    // us with 16, 64 and 256 lanes: 16384 tokens of 256 bf16 7.9, 12.0 and 31, of 512
    // 15.3, 16.8 and 33; 8192 of 2048 31, 27.8 and 28.2; 16 of 4096 22, 7.6 and 4.2
    const bool many = a.tokens >= 2048;
    if (a.per <= (many ? 64 : 16)) moe_combine_back_kernel<V, 16><<<grid(16), 256, 0, s>>>(a);
    else if (many || a.per <= 64) moe_combine_back_kernel<V, 64><<<grid(64), 256, 0, s>>>(a);
    else moe_combine_back_kernel<V, 256><<<grid(256), 256, 0, s>>>(a);
  });
}

}  // namespace qc
