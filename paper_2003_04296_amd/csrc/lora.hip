// lora.hip -- low-rank adapters of many requests beside a shared projection, and
// their gradients.  Token t of adapter g:
//   mid[t] = x[t] a_g^T            (rank values, fp32)
//   out[t] = y[t] + s_g mid[t] b_g^T
//   p[t]   = gy[t] b_g             (rank values, fp32)
//   gx[t]  = s_g p[t] a_g,  ga_g = s_g sum_t p[t] x[t],  gb_g = s_g sum_t gy[t] mid[t]
// An adapter's tokens are order[offsets[g]] .. order[offsets[g + 1] - 1], wherever
// they lie in the batch: a block takes 16 or 32 of them ("piece") and reads their
// rows in place.  Bound by HBM: the tokens' rows and the adapters in use are read
// once, which the matrix instructions keep up with at every rank.
//
// mid and p stay in fp32 between the passes.  Where they are an operand they enter
// as two bf16 parts, the leading 16 bits of each value: rounding them to the
// tensors' type would lose half of a 16-bit result's accuracy again, and in fp16
// overflow past 65504.  fp16 tensors that meet them are split, too, exactly: 11
// bits are a bf16 and a rest of 3.  The third product of that (of both rests) is
// below 2^-17 of the first and left out.
#include "dense_gemm.h"
#include "moe.h"
#include "moe_groups.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// A weight of each group, inner dimension contiguous.
struct GroupWeight {
  const uint16_t* p;
  int64_t ld, step;  // of rows and of groups
};

struct LoraArgs {
  Groups g;
  const int* order;
  const float* scale;  // [groups] or NULL
  int rank, len;       // len: the tokens' row length
  const uint16_t* x;   // rows of tokens: the operand (shrink, grad), what is added to or NULL (expand)
  int64_t ld_x;
  GroupWeight w;       // shrink [rank][len], expand [len][rank]
  float* mid;          // [parts][rows][ld_mid]
  int ld_mid, parts;
  int tiles;           // shrink: of ranks; expand and grad: of columns
  uint16_t* out;       // expand: rows of tokens; grad: [groups][rank][len] or [groups][len][rank]
  int64_t ld_out;
  float* part;         // grad: sums of pieces
  int64_t ld_part;
  int size;            // grad: rows of a piece
};

// The token of row r of the order; `m` tokens exist.
__device__ __forceinline__ int token_at(const LoraArgs& a, int r) {
  const int t = a.order[r];
  return (uint32_t)t < (uint32_t)a.g.rows ? t : -1;
}

// Eight values without the first k of them (0 <= k <= 8), zeros behind.
__device__ __forceinline__ v4u drop(v4u v, int k) {
  const uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  const int s = 16 * (k & 3);
  const uint64_t up = s ? hi << (64 - s) : 0;
  const uint64_t a = k >= 8 ? 0 : k >= 4 ? hi >> s : lo >> s | up, b = k >= 4 ? 0 : hi >> s;
  return v4u{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
}
// load8_first at the end of a row of `len` values, n of which begin at p, in one load
// (value by value, each would be waited for): the row's last eight, moved.
__device__ __forceinline__ v4u load8_end(const uint16_t* p, int n, int len) {
  if (len < 8) return load8_first(p, n);
  const int64_t d = n < 8 ? 8 - (int64_t)n : 0;
  return drop(load8(p - d), d < 8 ? (int)d : 8);
}
// load8_first inside contiguous memory that ends at `end`, `all` values long: what
// follows the n values is read and cleared.
__device__ __forceinline__ v4u load8_inside(const uint16_t* p, int n, const uint16_t* end, int64_t all) {
  if (all < 8) return load8_first(p, n);
  const int64_t d = p + 8 > end ? p + 8 - end : 0;
  v4u v = drop(load8(p - d), d < 8 ? (int)d : 8);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = n >= 2 * e + 2 ? v[e] : n == 2 * e + 1 ? v[e] & 0xFFFF : 0;
  return v;
}

// ---------------------------------------------------------------------------
// mid (and p): sums over a row's length
// ---------------------------------------------------------------------------

// A block takes MR * 16 tokens by RT * 16 ranks; its waves, and the blocks of a
// split product, take every so many-th 128 values of the rows, and are joined
// through LDS (splits by whoever reads mid).  Bound by reading x, 8192 tokens of 4096
// bf16 at rank 32 in 21.6 us (3.1 TB/s; 31 while each load was waited for), and by its
// latencies at few tokens (offsets, order, rows, the join): one token 4.0 us.
template <class T, int MR, int RT, int NW>
__device__ __forceinline__ void shrink(const LoraArgs& a, int e, int first, int here, int tile, int split,
                                       v4f (&part)[NW][MR * 16][RT * 4]) {
  constexpr int C = RT * 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, o = lane >> 4;
  // in place of rows past the piece its first one, of ranks past the last that one: their sums go nowhere
  const uint16_t *x[MR], *w[RT];
#pragma unroll
  for (int j = 0; j < MR; ++j) {
    const int t = token_at(a, first + (j * 16 + r < here ? j * 16 + r : 0));
    x[j] = a.x + (int64_t)(t < 0 ? 0 : t) * a.ld_x + o * 8;
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int c = tile * C + i * 16 + r;
    w[i] = a.w.p + e * a.w.step + (c < a.rank ? c : a.rank - 1) * a.w.ld + o * 8;
  }
  v4f acc[MR][RT];
#pragma unroll
  for (int j = 0; j < MR; ++j)
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // The next 128 values are on their way while these are multiplied.  The fence
  // keeps the loads ahead of the products: left alone, the compiler puts each right
  // before its use to save registers, and the wave waits for one at a time.
  const int blocks = a.len / 128, step = a.parts * NW;
  int b = split * NW + wave;
  struct Block {
    v4u x[MR][4], w[RT][4];
  } next;
  auto load = [&](int64_t k) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int j = 0; j < MR; ++j) next.x[j][s] = load8(x[j] + k + s * 32);
#pragma unroll
      for (int i = 0; i < RT; ++i) next.w[i][s] = load8(w[i] + k + s * 32);
    }
  };
  if (b < blocks) load((int64_t)b * 128);
  for (; b < blocks; b += step) {
    const Block now = next;
    if (b + step < blocks) load((int64_t)(b + step) * 128);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < MR; ++j)
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[j][i] = T::mfma(now.w[i][s], now.x[j][s], acc[j][i]);
  }
  if (b == blocks) {
    for (int k = blocks * 128; k < a.len; k += 32) {
      const int left = a.len - k - o * 8;
      v4u xf[MR], wf[RT];
#pragma unroll
      for (int j = 0; j < MR; ++j) xf[j] = a.len - k >= 32 ? load8(x[j] + k) : load8_end(x[j] + k, left, a.len);
#pragma unroll
      for (int i = 0; i < RT; ++i) wf[i] = a.len - k >= 32 ? load8(w[i] + k) : load8_end(w[i] + k, left, a.len);
#pragma unroll
      for (int j = 0; j < MR; ++j)
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[j][i] = T::mfma(wf[i], xf[j], acc[j][i]);
    }
  }
#pragma unroll
  for (int j = 0; j < MR; ++j)
#pragma unroll
    for (int i = 0; i < RT; ++i) part[wave][j * 16 + r][i * 4 + o] = acc[j][i];
  __syncthreads();
}
// The sum of a row's ranks [c * 4, + 4), after shrink.
template <int R, int C, int NW>
__device__ __forceinline__ v4f shrink_sum(const v4f (&part)[NW][R][C], int row, int c) {
  v4f s = part[0][row][c];
#pragma unroll
  for (int v = 1; v < NW; ++v) s += part[v][row][c];
  return s;
}

template <class T, int MR, int RT, int NW>
__global__ __launch_bounds__(NW * 64) void lora_shrink_kernel(LoraArgs a) {
  constexpr int R = MR * 16, C = RT * 16;
  __shared__ v4f part[NW][R][C / 4];
  const GroupPieces pieces(a.g, R);
  const int split = blockIdx.x % a.parts, tile = blockIdx.x / a.parts % a.tiles, p = blockIdx.x / a.parts / a.tiles;
  if (p >= pieces.total) return;
  int e, piece;
  pieces.find(a.g, p, e, piece);
  const GroupRows rows = group_rows(a.g, e);
  const int first = rows.first + piece * R, here = rows.count - piece * R < R ? rows.count - piece * R : R;
  shrink<T, MR, RT, NW>(a, e, first, here, tile, split, part);
  for (int i = threadIdx.x; i < here * (C / 4); i += NW * 64) {
    const int row = i / (C / 4), c = i % (C / 4);
    if (tile * C + c * 4 < a.ld_mid)
      *(v4f*)(a.mid + ((int64_t)split * a.g.rows + first + row) * a.ld_mid + tile * C + c * 4) =
          shrink_sum(part, row, c);
  }
}

// Joins the parts of mid into the first.
__global__ __launch_bounds__(256) void lora_join_kernel(float* mid, int64_t n, int parts, float* to) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n / 4; i += (int64_t)gridDim.x * 256) {
    v4f s = *(const v4f*)(mid + i * 4);
    for (int p = 1; p < parts; ++p) s += *(const v4f*)(mid + p * n + i * 4);
    *(v4f*)(to + i * 4) = s;
  }
}

// ---------------------------------------------------------------------------
// Two bf16 parts of a value
// ---------------------------------------------------------------------------

struct Two {
  uint16_t hi, lo;
};
__device__ __forceinline__ Two two_parts(float v) {
  const uint16_t hi = BF16::down(v);
  // an infinity has no rest
  return {hi, (hi & 0x7F80) == 0x7F80 ? (uint16_t)0 : BF16::down(v - BF16::up(hi))};
}
// Eight values of a tensor's type in bf16: itself, or a value and the rest (fp16).
template <class T>
__device__ __forceinline__ void in_bf16(v4u v, v4u out[2]) {
  if constexpr (T::REST) {  // bf16
    out[0] = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const Two a = two_parts(T::up((uint16_t)v[e])), b = two_parts(T::up((uint16_t)(v[e] >> 16)));
      out[0][e] = a.hi | (uint32_t)b.hi << 16;
      out[1][e] = a.lo | (uint32_t)b.lo << 16;
    }
  }
}
template <class T>
constexpr int BF16_PARTS = T::REST ? 1 : 2;

// ---------------------------------------------------------------------------
// out = y + s mid w^T
// ---------------------------------------------------------------------------

// A block takes MR * 16 tokens; a wave 64 columns at a time.  The 16 rows of
// operand i are columns (q / 4) * 16 + i * 4 + q % 4 of the 64, so that a lane
// ends up with 16 columns in a row, which it reads and writes 16 bytes at a time.
// Bound by HBM: 8192 tokens x 4096 bf16 read and written in 33 us (4.1 TB/s), gx of as
// many, written alone, in 24; by latencies at few tokens, one token 5.0 us.
// Tokens of no adapter: a copy, or zeros.  Rows [row0, + R) of the order, by `waves`
// waves, of which this is number `wave` of the columns' (`step` of them).
template <int R>
__device__ __forceinline__ void pass_rows(const LoraArgs& a, int64_t number, int first_chunk, int step) {
  const int lane = threadIdx.x & 63, chunks = (a.len + 63) / 64;
  const int end = a.g.offsets[a.g.n], begin = end < 0 ? 0 : end;
  const int64_t row0 = (int64_t)begin + number * R;
  if (row0 >= a.g.rows || a.x == a.out) return;
  for (int c = first_chunk; c < chunks; c += step)
    for (int j = 0; j < R; j += 8) {
      const int row = j + lane / 8, col = c * 64 + lane % 8 * 8;
      if (row0 + row >= a.g.rows || col >= a.len) continue;
      const int t = token_at(a, (int)row0 + row);
      if (t < 0) continue;
      const v4u v = a.x ? load8_first(a.x + t * a.ld_x + col, a.len - col) : v4u{0, 0, 0, 0};
      uint16_t* to = a.out + t * a.ld_out + col;
      if (col + 8 <= a.len) {
        reinterpret_cast<U128*>(to)->v = v;
      } else {
        for (int q = 0; col + q < a.len; ++q) to[q] = (uint16_t)(v[q / 2] >> (16 * (q & 1)));
      }
    }
}

// mid's values [c, c + 4) of a row of the second product's operand in LDS (zeros past
// the rank): rows of `steps` * 4 chunks of hi, as many of lo, and one to spread the banks.
__device__ __forceinline__ void put_mid(v4u* lds, int steps, int row, int c, int rank, v4f s) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (c + q >= rank) s[q] = 0.0f;
  const Two t[4] = {two_parts(s[0]), two_parts(s[1]), two_parts(s[2]), two_parts(s[3])};
  v2u* to = (v2u*)(lds + row * (steps * 8 + 1)) + c / 4;
  to[0] = v2u{t[0].hi | (uint32_t)t[1].hi << 16, t[2].hi | (uint32_t)t[3].hi << 16};
  to[steps * 8] = v2u{t[0].lo | (uint32_t)t[1].lo << 16, t[2].lo | (uint32_t)t[3].lo << 16};
}

// A wave's columns of a piece: chunks of 64 from `ch` on, every `step`-th.  start()
// puts the first loads under way, run() needs the operand in LDS.
template <class T, int MR>
struct Columns {
  const LoraArgs& a;
  int r, o, steps, chunks;
  const uint16_t *wp, *w_end;
  int token[MR];
  v4u y[MR][2], wf[4];
  float scale;

  __device__ __forceinline__ Columns(const LoraArgs& args, int e, int first, int here) : a(args) {
    const int lane = threadIdx.x & 63;
    r = lane & 15;
    o = lane >> 4;
    steps = (a.rank + 31) / 32;
    chunks = (a.len + 63) / 64;
    wp = a.w.p + e * a.w.step;
    w_end = a.w.p + a.g.n * a.w.step;
    scale = a.scale ? a.scale[e] : 1.0f;
#pragma unroll
    for (int j = 0; j < MR; ++j) {
      token[j] = j * 16 + r < here ? token_at(a, first + j * 16 + r) : -1;
      y[j][0] = y[j][1] = v4u{0, 0, 0, 0};
    }
  }
  // Loads are the same for every lane where a chunk of columns exists whole, from a
  // row that exists where the lane has none, so that they can be under way together:
  // those of the next 64 columns (and of the next 32 ranks) while these are multiplied.
  __device__ __forceinline__ void load_w(int ch, int k) {
    const int c0 = ch * 64 + (r >> 2) * 16 + (r & 3), at = k * 32 + o * 8;
    if (a.rank % 8 == 0) {
      const bool in = at < a.rank;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + i * 4 < a.len ? c0 + i * 4 : a.len - 1;
        wf[i] = load8(wp + c * a.w.ld + (in ? at : 0));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) wf[i] = in ? wf[i] : v4u{0, 0, 0, 0};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + i * 4 < a.len ? c0 + i * 4 : a.len - 1;
        wf[i] = load8_inside(wp + c * a.w.ld + (at < a.rank ? at : 0), a.rank - at, w_end, a.g.n * a.w.step);
      }
    }
  }
  __device__ __forceinline__ void load_y(int ch) {
    if (!a.x) return;
    const int c = ch * 64 + o * 16;
#pragma unroll
    for (int j = 0; j < MR; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint16_t* from = a.x + (token[j] < 0 ? 0 : token[j]) * a.ld_x;
        y[j][h] = ch * 64 + 64 <= a.len ? load8(from + c + h * 8) : load8_end(from + c + h * 8, a.len - c - h * 8, a.len);
      }
  }
  __device__ __forceinline__ void start(int ch) {
    if (ch < chunks) {
      load_w(ch, 0);
      load_y(ch);
    }
  }
  __device__ __forceinline__ void run(const v4u* lds, int ch, int step) {
    const int ld = steps * 8 + 1;
    v4f acc[MR][4];
#pragma unroll
    for (int j = 0; j < MR; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    v4u base[MR][2];
    for (int k = 0; ch < chunks;) {
      v4u w[4][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) in_bf16<T>(wf[i], w[i]);
      if (k == 0) {
#pragma unroll
        for (int j = 0; j < MR; ++j) base[j][0] = y[j][0], base[j][1] = y[j][1];
      }
      const int here_ch = ch, here_k = k;
      if (++k == steps) {
        k = 0;
        ch += step;
      }
      if (ch < chunks) {
        load_w(ch, k);
        if (k == 0) load_y(ch);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < MR; ++j) {
        const v4u* s = lds + (j * 16 + r) * ld + here_k * 4 + o;
        const v4u hi = s[0], lo = s[steps * 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[j][i] = BF16::mfma(w[i][0], hi, acc[j][i]);
          acc[j][i] = BF16::mfma(w[i][0], lo, acc[j][i]);
          if constexpr (BF16_PARTS<T> == 2) acc[j][i] = BF16::mfma(w[i][1], hi, acc[j][i]);
        }
      }
      if (k != 0) continue;
      const int mine = here_ch * 64 + o * 16;
#pragma unroll
      for (int j = 0; j < MR; ++j) {
        if (token[j] >= 0) {
          uint16_t* to = a.out + token[j] * a.ld_out + mine;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint16_t v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q)
              v[q] = T::down(fmaf(scale, acc[j][h * 2 + q / 4][q % 4], T::up((uint16_t)(base[j][h][q / 2] >> (16 * (q & 1))))));
            if (mine + h * 8 + 8 <= a.len) {
              reinterpret_cast<U128*>(to + h * 8)->v =
                  v4u{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16,
                      v[6] | (uint32_t)v[7] << 16};
            } else {
#pragma unroll
              for (int q = 0; q < 8; ++q)
                if (mine + h * 8 + q < a.len) to[h * 8 + q] = v[q];
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
  }
};

template <class T, int MR>
__global__ __launch_bounds__(256) void lora_expand_kernel(LoraArgs a) {
  constexpr int R = MR * 16;
  extern __shared__ v4u lds[];
  const GroupPieces pieces(a.g, R);
  const int tile = blockIdx.x % a.tiles, p = blockIdx.x / a.tiles;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (p >= pieces.total) return pass_rows<R>(a, p - pieces.total, tile * 4 + wave, a.tiles * 4);
  int e, piece;
  pieces.find(a.g, p, e, piece);
  const GroupRows rows = group_rows(a.g, e);
  const int first = rows.first + piece * R, here = rows.count - piece * R < R ? rows.count - piece * R : R;
  Columns<T, MR> columns(a, e, first, here);
  columns.start(tile * 4 + wave);
  const int steps = columns.steps;
  for (int i = threadIdx.x; i < R * steps * 8; i += 256) {
    const int row = i / (steps * 8), c = i % (steps * 8) * 4;
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (row < here && c < a.rank) {
      const float* m = a.mid + (int64_t)(first + row) * a.ld_mid + c;
      s = *(const v4f*)m;
#pragma unroll 4
      for (int q = 1; q < a.parts; ++q) s += *(const v4f*)(m + (int64_t)q * a.g.rows * a.ld_mid);
    }
    put_mid(lds, steps, row, c, a.rank, s);
  }
  __syncthreads();
  columns.run(lds, tile * 4 + wave, a.tiles * 4);
}

// Both products of few tokens in one launch: a block sums mid by itself, as every
// block of the piece's columns does (the adapter's a then comes from L2).  Bound by its
// latencies: offsets, order, rows, the join of the waves, the second product.
template <class T, int RT, int NW>
__global__ __launch_bounds__(NW * 64) void lora_few_kernel(LoraArgs in, LoraArgs a) {
  constexpr int R = 16, C = RT * 16, STEPS = (RT + 1) / 2;
  __shared__ v4f part[NW][R][C / 4];
  __shared__ v4u lds[R * (STEPS * 8 + 1)];
  const GroupPieces pieces(a.g, R);
  const int tile = blockIdx.x % a.tiles, p = blockIdx.x / a.tiles;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ch = tile * NW + wave;
  if (p >= pieces.total) return pass_rows<R>(a, p - pieces.total, ch, a.tiles * NW);
  int e, piece;
  pieces.find(a.g, p, e, piece);
  const GroupRows rows = group_rows(a.g, e);
  const int first = rows.first + piece * R, here = rows.count - piece * R < R ? rows.count - piece * R : R;
  Columns<T, 1> columns(a, e, first, here);
  columns.start(ch);
  shrink<T, 1, RT, NW>(in, e, first, here, 0, 0, part);
  for (int i = threadIdx.x; i < R * columns.steps * 8; i += NW * 64) {
    const int row = i / (columns.steps * 8), c = i % (columns.steps * 8);
    const bool on = row < here && c * 4 < a.rank;
    const v4f s = on ? shrink_sum(part, row, c) : v4f{0.0f, 0.0f, 0.0f, 0.0f};
    if (on && tile == 0 && in.mid) *(v4f*)(in.mid + (int64_t)(first + row) * in.ld_mid + c * 4) = s;
    put_mid(lds, columns.steps, row, c * 4, a.rank, s);
  }
  __syncthreads();
  columns.run(lds, ch, a.tiles * NW);
}

// ---------------------------------------------------------------------------
// Weight gradients: sums over an adapter's tokens
// ---------------------------------------------------------------------------

// Rows of an adapter are taken `size` at a time; a block has 256 columns of a
// piece and 64 ranks.  The sums of an adapter with one piece (or none: zeros) are
// results; others go to part.
constexpr int GRAD_MOST = 512;  // rows of a piece, a multiple of 32

// Writes 4 values of a row of a gradient.
template <class T>
__device__ __forceinline__ void put_grad(const LoraArgs& a, int e, int rows, int cols, int row, int col, v4f v) {
  const float s = a.scale ? a.scale[e] : 1.0f;
  uint16_t* to = a.out + ((int64_t)e * rows + row) * cols + col;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (col + q < cols) to[q] = T::down(s * v[q]);
}

// Results [rank][len] (ga), or with FLIP [len][rank] (gb).  Both operands run down
// their columns: they pass through registers into LDS rows of one token and are
// read transposed.  Bound by HBM and by the sums' start: 8192 tokens x 4096 bf16 at
// rank 32 in 27 us (2.5 TB/s), three blocks a unit.
template <class T, int RT, bool FLIP>
__global__ __launch_bounds__(256, RT == 4 ? 2 : 3) void lora_grad_kernel(LoraArgs a) {
  constexpr int C = 256, XCH = 32 * C / 8, SCH = 32 * 128 / 8, STAGE = XCH + SCH;
  [[maybe_unused]] __shared__ v4u store[2 * STAGE];
  [[maybe_unused]] __shared__ int tokens[GRAD_MOST + 64];  // and two stages of none
#ifdef __HIP_DEVICE_COMPILE__
  lds_v4u* const lds = (lds_v4u*)store;
  const GroupPieces pieces(a.g, a.size, true);
  const int rts = (a.rank + 63) / 64;
  const int tile = blockIdx.x % a.tiles, rt = blockIdx.x / a.tiles % rts, p = blockIdx.x / a.tiles / rts;
  if (p >= pieces.total) return;
  int e, piece;
  pieces.find(a.g, p, e, piece);
  const GroupRows rows = group_rows(a.g, e);
  const int first = rows.first + piece * a.size;
  const int here = rows.count - piece * a.size < a.size ? rows.count - piece * a.size : a.size;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = tile * C, r0 = rt * 64;
  v4f acc[4][RT];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = threadIdx.x; i < GRAD_MOST + 64; i += 256) tokens[i] = i < here ? token_at(a, first + i) : -1;
  __syncthreads();
  // A stage: 32 tokens.  Of x a thread has 4 chunks of 8 columns, of mid 2 x 4 ranks.
  // Two stages are on their way while one is multiplied.
  v4u xr[4], xr2[4];
  v4f sr[2], sr2[2];
  const int xc = threadIdx.x % 32, sc = threadIdx.x % 16 * 4;
  const bool whole_cols = c0 + C <= a.len, rank_in = r0 + sc < a.rank;
  auto load = [&](int at) {
    int t[4], u[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = tokens[at + threadIdx.x / 32 + i * 8];
#pragma unroll
    for (int i = 0; i < 2; ++i) u[i] = tokens[at + threadIdx.x / 16 + i * 16];
    // in place of a token that is none the first one, which then counts for nothing
    const int col = c0 + xc * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t* from = a.x + (t[i] < 0 ? 0 : t[i]) * a.ld_x + col;
      xr2[i] = whole_cols ? load8(from) : load8_end(from, a.len - col, a.len);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = at + threadIdx.x / 16 + i * 16;
      sr2[i] = *(const v4f*)(a.mid + (int64_t)(first + (u[i] >= 0 ? k : 0)) * a.ld_mid + (rank_in ? r0 + sc : 0));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) xr2[i] = t[i] >= 0 ? xr2[i] : v4u{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) sr2[i] = u[i] >= 0 && rank_in ? sr2[i] : v4f{0.0f, 0.0f, 0.0f, 0.0f};
  };
  auto advance = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i) xr[i] = xr2[i];
#pragma unroll
    for (int i = 0; i < 2; ++i) sr[i] = sr2[i];
  };
  auto put = [&](lds_v4u* to) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = threadIdx.x / 32 + i * 8;
      to[k * (C / 8) + (xc ^ swz_col(k))] = xr[i];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = threadIdx.x / 16 + i * 16;
      const Two t[4] = {two_parts(sr[i][0]), two_parts(sr[i][1]), two_parts(sr[i][2]), two_parts(sr[i][3])};
      lds_v4u* const row = to + XCH + k * 16;
      typedef __attribute__((address_space(3))) v2u* half;
      ((half)(row + ((sc / 8) ^ swz_col(k))))[sc / 4 & 1] =
          v2u{t[0].hi | (uint32_t)t[1].hi << 16, t[2].hi | (uint32_t)t[3].hi << 16};
      ((half)(row + ((sc / 8 + 8) ^ swz_col(k))))[sc / 4 & 1] =
          v2u{t[0].lo | (uint32_t)t[1].lo << 16, t[2].lo | (uint32_t)t[3].lo << 16};
    }
  };
  if (here > 0) {
    load(0);
    advance();
    load(32);
    put(lds);
    advance();
  }
  for (int at = 0, b = 0; at < here; at += 32, b ^= 1) {
    __syncthreads();
    const lds_v4u* now = lds + b * STAGE;
    if (at + 64 < here) load(at + 64);
    __builtin_amdgcn_sched_barrier(0);
    v4u s[2][RT];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < RT; ++j) s[h][j] = fragment<32, 128, true>(now + XCH, h * 64 + j * 16, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v4u x[2];
      in_bf16<T>(fragment<32, C, true>(now, wave * 64 + i * 16, 0), x);
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        auto add = [&](v4u xf, v4u sf) {
          acc[i][j] = FLIP ? BF16::mfma(sf, xf, acc[i][j]) : BF16::mfma(xf, sf, acc[i][j]);
        };
        add(x[0], s[0][j]);
        add(x[0], s[1][j]);
        if constexpr (BF16_PARTS<T> == 2) add(x[1], s[0][j]);
      }
    }
    if (at + 32 < here) put(lds + (b ^ 1) * STAGE);
    advance();
  }
  const bool whole = rows.count <= a.size;
  const int nr = FLIP ? a.len : a.rank, nc = FLIP ? a.rank : a.len;
  float* const to = a.part + group_part(rows.first, piece, a.size) * nr * a.ld_part;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int x = c0 + wave * 64 + i * 16, s = r0 + j * 16;  // the first column and rank
      const int row = (FLIP ? x : s) + (lane & 15), col = (FLIP ? s : x) + (lane >> 4) * 4;
      if (row >= nr || col >= nc) continue;
      if (whole) put_grad<T>(a, e, nr, nc, row, col, acc[i][j]);
      else *(v4f*)(to + (int64_t)row * a.ld_part + col) = acc[i][j];
    }
#endif
}

// Joins the pieces of the adapters that have several: the y-th of them.
template <class T, bool FLIP>
__global__ __launch_bounds__(256) void lora_grad_join_kernel(LoraArgs a) {
  const GroupPieces several(a.g, a.size, false, true);
  if ((int)blockIdx.y >= several.total) return;
  int e, unused;
  several.find(a.g, blockIdx.y, e, unused);
  const GroupRows rows = group_rows(a.g, e);
  const int n = (rows.count - 1) / a.size + 1;
  const int nr = FLIP ? a.len : a.rank, nc = FLIP ? a.rank : a.len, per = (int)(a.ld_part / 4);
  const int64_t all = (int64_t)nr * per, plane = nr * a.ld_part;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int row = (int)(i / per), col = (int)(i % per) * 4;
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int p = 0; p < n; ++p) s += *(const v4f*)(a.part + group_part(rows.first, p, a.size) * plane + row * a.ld_part + col);
    put_grad<T>(a, e, nr, nc, row, col, s);
  }
}

// Transposed copies of each group's matrix [rows][cols], in rows of ld_out: of b, and
// of a where blocks are left for it.
struct Transpose {
  const uint16_t* w[2];
  uint16_t* out[2];
  int rows[2], cols[2];
  int64_t ld_out[2];
  uint32_t blocks;  // of the first
};
__global__ __launch_bounds__(256) void lora_transpose_kernel(Transpose a) {
  __shared__ uint16_t t[64][66];
  const int which = blockIdx.x >= a.blocks;
  const uint32_t id = blockIdx.x - (which ? a.blocks : 0);
  const int rows = a.rows[which], cols = a.cols[which], tr_n = (rows + 63) / 64, tc_n = (cols + 63) / 64;
  const int tc = id % tc_n, tr = id / tc_n % tr_n;
  const int64_t g = id / tc_n / tr_n;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  uint16_t v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = tr * 64 + y + i * 4, c = tc * 64 + x;
    v[i] = r < rows && c < cols ? a.w[which][(g * rows + r) * cols + c] : (uint16_t)0;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) t[y + i * 4][x] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = tr * 64 + x, c = tc * 64 + y + i * 4;
    if (r < rows && c < cols) a.out[which][(g * cols + c) * a.ld_out[which] + r] = t[x][y + i * 4];
  }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------

int ld_mid(const qconv_lora_desc& d) { return (int)round_up(d.rank, 4); }
size_t mid_bytes(const qconv_lora_desc& d) { return (size_t)round_up((int64_t)d.m * ld_mid(d) * 4, 16); }

// Tokens of a piece.  With 32 the adapters are read half as often, with 16 twice as
// many blocks share the chip.  us of a forward of 4096 -> 4096 with 16 and 32: rank 16,
// 4096 tokens of 4 adapters 30.4 and 36.0, 8192 of 64 53.9 and 47.9; rank 64, 2048
// tokens 40.9 and 31.3, 8192 96.8 and 69.4.
int piece_rows(const qconv_lora_desc& d) { return d.m >= (d.rank > 32 ? 2048 : 8192) ? 32 : 16; }

// Blocks that share the sums over a row of `len` values: until there are about
// 512 of them, as long as each wave has 128 values (one token of 4096 inputs: 8.5 us of
// a forward with 4 blocks, 11.3 with one).
int shrink_parts(const qconv_lora_desc& d, int len) {
  const int R = piece_rows(d);
  const int64_t blocks = GroupPieces::most(d.m, d.groups, R) * ceil_div(d.rank, 64);
  int64_t parts = 512 / (blocks > 0 ? blocks : 1);
  if (parts > len / 1024) parts = len / 1024;
  return parts < 1 ? 1 : parts > 8 ? 8 : (int)parts;
}

constexpr int NW = 8;

template <class T, int MR, int RT>
int run_shrink_t(LoraArgs& a, hipStream_t s) {
  a.tiles = ceil_div(a.rank, RT * 16);
  const int64_t blocks = GroupPieces::most(a.g.rows, a.g.n, MR * 16) * a.tiles * a.parts;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  lora_shrink_kernel<T, MR, RT, NW><<<(unsigned)blocks, NW * 64, 0, s>>>(a);
  return hip_status();
}
template <class T>
int run_shrink(LoraArgs& a, int rows, hipStream_t s) {
  if (rows == 32)
    return a.rank <= 16 ? run_shrink_t<T, 2, 1>(a, s) : a.rank <= 32 ? run_shrink_t<T, 2, 2>(a, s) : run_shrink_t<T, 2, 4>(a, s);
  return a.rank <= 16 ? run_shrink_t<T, 1, 1>(a, s) : a.rank <= 32 ? run_shrink_t<T, 1, 2>(a, s) : run_shrink_t<T, 1, 4>(a, s);
}

template <class T>
int run_expand(LoraArgs& a, int rows, hipStream_t s) {
  const int64_t pieces = a.g.rows / rows + (a.g.n + 1 < a.g.rows ? a.g.n + 1 : a.g.rows);
  // a block per 256 columns while there are at most about 1024: more read an adapter's
  // offsets and mid for fewer columns each (rank 16, 4096 -> 8192, us of a forward with
  // 512, 1024 and 2048: 13.6, 13.0 and 14.2 for 512 tokens, 30.5, 28.3 and 29.2 for 2048)
  const int64_t most = ceil_div(a.len, 256), want = 1024 / pieces;
  a.tiles = (int)(want < 1 ? 1 : want < most ? want : most);
  if (pieces * a.tiles >= (1 << 23)) return QCONV_EUNSUPPORTED;
  const size_t lds = (size_t)rows * (ceil_div(a.rank, 32) * 8 + 1) * 16;
  const unsigned blocks = (unsigned)(pieces * a.tiles);
  if (rows == 32) lora_expand_kernel<T, 2><<<blocks, 256, lds, s>>>(a);
  else lora_expand_kernel<T, 1><<<blocks, 256, lds, s>>>(a);
  return hip_status();
}

// The tokens that one launch serves: sums that are short, or few tokens, for which the
// second launch costs the host as much (4.5 us) as the kernels differ.  us on the device
// in one launch and in two (in a graph): 1024 -> 1024 at rank 16 5.6 and 7.9 for one token, 7.2 and
// 9.3 for 1024 tokens of 40 adapters, at rank 64 10.1 and 11.8, 12.5 and 13.4; 4096 -> 4096 at
// rank 16 9.0 and 8.5 for one token, 12.2 and 9.9 for 64 of 40, at rank 64 21 and 12.8.
// Sixteen waves a block instead of eight: 9.9 in place of 9.0.
constexpr int FEW_BLOCKS = 256;
bool few_tokens(const qconv_lora_desc& d) {
  if (d.rank > 64) return false;
  const int64_t pieces = GroupPieces::most(d.m, d.groups, 16), ranks = d.rank <= 16 ? 1 : d.rank <= 32 ? 2 : 4;
  return (d.k <= 1024 && pieces <= 128) || (d.k * ranks <= 4096 && pieces <= 16);
}

template <class T>
int run_few(LoraArgs& in, LoraArgs& a, hipStream_t s) {
  const int64_t pieces = a.g.rows / 16 + (a.g.n + 1 < a.g.rows ? a.g.n + 1 : a.g.rows);
  const int64_t most = ceil_div(a.len, 64 * NW), want = FEW_BLOCKS / pieces;
  a.tiles = (int)(want < 1 ? 1 : want < most ? want : most);
  const unsigned blocks = (unsigned)(pieces * a.tiles);
  if (a.rank <= 16) lora_few_kernel<T, 1, NW><<<blocks, NW * 64, 0, s>>>(in, a);
  else if (a.rank <= 32) lora_few_kernel<T, 2, NW><<<blocks, NW * 64, 0, s>>>(in, a);
  else lora_few_kernel<T, 4, NW><<<blocks, NW * 64, 0, s>>>(in, a);
  return hip_status();
}

// Tokens of a piece of a weight gradient: as many as make about 1024 blocks (8192
// tokens x 4096 at rank 32: 27 us and 7.6 of the join; with 600 blocks 34 and 5.7).
int grad_rows(const LoraArgs& a, int len) {
  const int64_t n = (int64_t)a.g.rows * ceil_div(len, 256) * ceil_div(a.rank, 64) / 1024;
  return n < 128 ? 128 : n < GRAD_MOST ? (int)round_up(n, 32) : GRAD_MOST;
}
size_t grad_bytes(const qconv_lora_desc& d) {
  size_t most = 0;
  LoraArgs a = {};
  a.g.rows = d.m;
  a.rank = d.rank;
  for (int len : {d.k, d.n}) {
    const int64_t size = grad_rows(a, len), p = len == d.k ? d.rank * round_up(len, 4) : 0, q = len == d.n ? len * round_up(d.rank, 4) : 0;
    const size_t bytes = d.m > size ? (size_t)(2 * ((d.m + size - 1) / size) * (p > q ? p : q) * 4) : 0;
    most = bytes > most ? bytes : most;
  }
  return most;
}
template <class T, int RT, bool FLIP>
int run_grad_t(LoraArgs& a, hipStream_t s) {
  a.size = grad_rows(a, a.len);
  a.tiles = ceil_div(a.len, 256);
  a.ld_part = round_up(FLIP ? a.rank : a.len, 4);
  const int64_t blocks = ((int64_t)a.g.rows / a.size + a.g.n) * a.tiles * ceil_div(a.rank, 64);
  if (blocks >= (1 << 23)) return QCONV_EUNSUPPORTED;
  lora_grad_kernel<T, RT, FLIP><<<(unsigned)blocks, 256, 0, s>>>(a);
  if (a.g.rows > a.size) {
    const int64_t n = (FLIP ? a.len : a.rank) * a.ld_part / 4;
    const int several = a.g.rows / a.size < a.g.n ? a.g.rows / a.size : a.g.n;
    const dim3 grid((unsigned)(n < (1 << 16) ? (n + 255) / 256 : 256), several);
    lora_grad_join_kernel<T, FLIP><<<grid, 256, 0, s>>>(a);
  }
  return hip_status();
}
template <class T, bool FLIP>
int run_grad(LoraArgs& a, hipStream_t s) {
  return a.rank <= 16 ? run_grad_t<T, 1, FLIP>(a, s) : a.rank <= 32 ? run_grad_t<T, 2, FLIP>(a, s) : run_grad_t<T, 4, FLIP>(a, s);
}

int run_transpose(const Transpose& t, int groups, bool both, hipStream_t s) {
  auto blocks = [&](int i) { return (int64_t)groups * ceil_div(t.rows[i], 64) * ceil_div(t.cols[i], 64); };
  if (blocks(0) + blocks(1) >= (1 << 23)) return QCONV_EUNSUPPORTED;
  Transpose a = t;
  a.blocks = (uint32_t)blocks(0);
  lora_transpose_kernel<<<(unsigned)(blocks(0) + (both ? blocks(1) : 0)), 256, 0, s>>>(a);
  return hip_status();
}

int run_join(float* parts, int n_parts, const qconv_lora_desc& d, float* to, hipStream_t s) {
  const int64_t n = (int64_t)d.m * ld_mid(d);
  lora_join_kernel<<<(unsigned)(n < (1 << 20) ? (n / 4 + 255) / 256 : 1024), 256, 0, s>>>(parts, n, n_parts, to);
  return hip_status();
}

template <class T>
int forward(const qconv_lora_desc& d, LoraArgs a, const void* x, const void* wa, const void* wb, const void* y, void* out,
            float* mid, void* ws, hipStream_t s) {
  const int rows = piece_rows(d);
  a.len = d.k;
  a.x = (const uint16_t*)x;
  a.ld_x = d.ld_x;
  a.w = {(const uint16_t*)wa, d.k, (int64_t)d.rank * d.k};
  LoraArgs b = a;
  b.len = d.n;
  b.x = (const uint16_t*)y;
  b.ld_x = d.ld_y;
  b.w = {(const uint16_t*)wb, d.rank, (int64_t)d.n * d.rank};
  b.out = (uint16_t*)out;
  b.ld_out = d.ld_out;
  if (few_tokens(d)) {
    a.mid = mid;
    return run_few<T>(a, b, s);
  }
  a.parts = shrink_parts(d, d.k);
  a.mid = a.parts == 1 && mid ? mid : (float*)ws;
  int rc = run_shrink<T>(a, rows, s);
  if (rc == QCONV_OK && mid && a.parts > 1) {
    rc = run_join(a.mid, a.parts, d, mid, s);
    a.mid = mid;
    a.parts = 1;
  }
  b.mid = a.mid;
  b.parts = a.parts;
  return rc ? rc : run_expand<T>(b, rows, s);
}

struct BackBytes {
  size_t bt, at, parts, p, grad;
};
BackBytes back_bytes(const qconv_lora_desc& d) {
  BackBytes b;
  b.bt = (size_t)round_up((int64_t)d.groups * d.rank * round_up(d.n, 8) * 2, 16);
  b.at = (size_t)round_up((int64_t)d.groups * d.k * round_up(d.rank, 8) * 2, 16);
  const int parts = shrink_parts(d, d.n);
  b.parts = parts > 1 ? parts * mid_bytes(d) : 0;
  b.p = mid_bytes(d);
  b.grad = grad_bytes(d);
  return b;
}

template <class T>
int backward(const qconv_lora_desc& d, LoraArgs a, const void* x, const void* wa, const void* wb, const float* mid,
             const void* gy, void* gx, void* ga, void* gb, void* ws, hipStream_t s) {
  const BackBytes b = back_bytes(d);
  uint16_t* bt = (uint16_t*)ws;
  uint16_t* at = (uint16_t*)((char*)bt + b.bt);
  float* parts = (float*)((char*)at + b.at);
  float* p = (float*)((char*)parts + b.parts);
  a.part = (float*)((char*)p + b.p);
  int rc = QCONV_OK;
  if (d.m > 0) {
    const int64_t ld_bt = round_up(d.n, 8), ld_at = round_up(d.rank, 8);
    rc = run_transpose({{(const uint16_t*)wb, (const uint16_t*)wa}, {bt, at}, {d.n, d.rank}, {d.rank, d.k}, {ld_bt, ld_at}, 0},
                       d.groups, gx != nullptr, s);
    if (rc) return rc;
    a.parts = shrink_parts(d, d.n);
    a.len = d.n;
    a.x = (const uint16_t*)gy;
    a.ld_x = d.ld_y;
    a.w = {bt, ld_bt, (int64_t)d.rank * ld_bt};
    a.mid = a.parts > 1 ? parts : p;
    rc = run_shrink<T>(a, piece_rows(d), s);
    if (rc) return rc;
    if (a.parts > 1) rc = run_join(parts, a.parts, d, p, s);
    if (rc) return rc;
    a.mid = p;
    a.parts = 1;
    if (gx) {
      a.len = d.k;
      a.x = nullptr;
      a.w = {at, ld_at, (int64_t)d.k * ld_at};
      a.out = (uint16_t*)gx;
      a.ld_out = d.k;
      rc = run_expand<T>(a, piece_rows(d), s);
      if (rc) return rc;
    }
  }
  if (ga) {
    a.mid = p;
    a.len = d.k;
    a.x = (const uint16_t*)x;
    a.ld_x = d.ld_x;
    a.out = (uint16_t*)ga;
    rc = run_grad<T, false>(a, s);
    if (rc) return rc;
    a.mid = (float*)mid;
    a.len = d.n;
    a.x = (const uint16_t*)gy;
    a.ld_x = d.ld_y;
    a.out = (uint16_t*)gb;
    rc = run_grad<T, true>(a, s);
  }
  return rc;
}

LoraArgs lora_args(const qconv_lora_desc& d, const int* offsets, const int* order, const float* scale) {
  LoraArgs a = {};
  a.g = {offsets, d.groups, d.m};
  a.order = order;
  a.scale = scale;
  a.rank = d.rank;
  a.ld_mid = ld_mid(d);
  a.parts = 1;
  return a;
}

}  // namespace

size_t lora_forward_bytes(const qconv_lora_desc& d, bool keep_mid) {
  if (few_tokens(d)) return 0;
  const int parts = shrink_parts(d, d.k);
  return keep_mid && parts == 1 ? 0 : parts * mid_bytes(d);
}

int launch_lora_forward(const qconv_lora_desc& d, const void* x, const void* wa, const void* wb, const int* offsets,
                        const int* order, const float* scale, const void* y, void* out, float* mid, void* ws,
                        hipStream_t s) {
  if (d.m == 0) return QCONV_OK;
  const LoraArgs a = lora_args(d, offsets, order, scale);
  return d.dtype == QCONV_F16 ? forward<F16>(d, a, x, wa, wb, y, out, mid, ws, s)
                              : forward<BF16>(d, a, x, wa, wb, y, out, mid, ws, s);
}

size_t lora_backward_bytes(const qconv_lora_desc& d) {
  const BackBytes b = back_bytes(d);
  return b.bt + b.at + b.parts + b.p + b.grad;
}

int launch_lora_backward(const qconv_lora_desc& d, const void* x, const void* wa, const void* wb, const int* offsets,
                         const int* order, const float* scale, const float* mid, const void* gy, void* gx, void* ga,
                         void* gb, void* ws, hipStream_t s) {
  const LoraArgs a = lora_args(d, offsets, order, scale);
  return d.dtype == QCONV_F16 ? backward<F16>(d, a, x, wa, wb, mid, gy, gx, ga, gb, ws, s)
                              : backward<BF16>(d, a, x, wa, wb, mid, gy, gx, ga, gb, ws, s);
}

}  // namespace qc
