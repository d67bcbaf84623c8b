// dense_gemm.h -- C[r][c] = sum_k R(r, k) Q(c, k) on the matrix cores for many
// rows: the three products of the feed-forward block in 16-bit types, and
// those with 4-bit weights for more tokens than dense_rows.h takes.
//
// Operands whose k runs along their rows ("row form": x, W in the forward,
// dg/du in gx) are read from LDS as 16 bytes per lane, operands whose k runs
// down their columns ("column form": W in gx, all of gW) through the
// transposing LDS reads.  4-bit weights are expanded on their way into LDS.
//
// Bound by the matrix cores at many tokens, by reading the operands at few.
// Measured in bf16, 4096 <-> 16384 features and 8192 tokens (2.2 TFLOP each), one
// pass after the other: forward 1.79 ms (1230 TFLOP/s; 2.12 with the 1.07 GB of
// pre, which leave at the memory's rate while the next tile waits), gx 1.67 ms
// (1315), both weight gradients 1.77 ms (1240).  A launch alone, before which the
// device was idle: 2.23 with pre, 1.68 and 1.91.  One library product of these
// sizes reaches 1335, 1195 and 1059 TFLOP/s in the three forms.
#pragma once

#include <type_traits>

#include "dense.h"
#include "qconv_internal.h"

namespace qc {

typedef __attribute__((address_space(3))) v4u lds_v4u;
typedef __attribute__((address_space(3))) void lds_void;

// Row form: value (r, k) at p[r * ld + k]; column form: at p[k * ld + r].
struct Operand {
  const uint16_t* p;
  int64_t ld;
};

enum GemmOut { OUT_GATED = 0, OUT_PLAIN = 1 };

struct GemmArgs {
  Operand r[2], c[2];  // by segment (the sums of gx run over two operand pairs) or by half (gW's two outputs)
  int rows, cols, k;   // C's extent (of one half) and the products of one segment
  int segments;        // 1 or 2
  int halves;          // 2: a second C from r[1] with the same c[0]
  int tiles_r, tiles_c;
  // 4-bit weights in place of c: codes, scales, and a power of two per row
  // that keeps scale * magnitude inside fp16 (NULL for bf16)
  const uint8_t* codes[2];
  const uint16_t* scales[2];
  const float* unit[2];
  int kp;  // codes per row
  void* out[2];
  int64_t ld_out;
  const float* bias;
  float* pre;  // OUT_GATED: [rows][2][ld_pre] or NULL
  int ld_pre;
  int act;
  // the products of a tile split over `parts` blocks: fp32 sums go to
  // part[parts][2 or halves][part_rows][ld_part] (NULL: to out), joined by
  // dense_join_kernel
  int parts;
  float* part;
  int part_rows, ld_part;
};

// LDS holds chunks of 16 bytes; a stage holds KS products (32 or 64) of every
// row.  Row form: rows of KS / 8 chunks, the chunk index xored by the row so
// that the 16 rows that 16 lanes read at one place lie in different banks.
// (16-byte reads are served 16 lanes at a time, 0-3, 12-15, 20-23 and 24-27,
// then 4-11, 16-19 and 28-31; r & 7 for rows of 8 chunks and the map 0, 2, 3, 1
// of r / 4 for rows of 4 keep both free of conflicts.)  Column form: one LDS
// row per product, of ROWS values; a transposing read touches 4 of them at one
// place, and the lanes beside it 4 more 8 rows below, which the xor spreads
// over the banks.
template <int KS>
__device__ __forceinline__ int swz_row(int r) {
  return KS == 64 ? r & 7 : ((r >> 2) & 1) << 1 ^ ((r >> 3) & 1) * 3;
}
__device__ __forceinline__ int swz_col(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) << 1; }

// Columns of the gated forward: 64 columns of the tile are 32 gate rows and
// the 32 up rows of the same hidden features, so that one lane ends up with
// both sums.  The weight row of tile column t.
template <bool PAIR>
__device__ __forceinline__ int weight_row(int t) {
  return PAIR ? (t / 64) * 32 + t % 32 : t;
}

// A pointer that is the same in every lane, in scalar registers.  (Where other
// code of the loop diverges, the compiler loses sight of that and loads lane
// group by lane group.)
__device__ __forceinline__ const uint16_t* uniform(const uint16_t* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const uint16_t*)((uint64_t)hi << 32 | lo);
}

// The tile of one 16-bit operand: ROWS rows (or columns) of C by KS
// products, staged by NT threads, CH chunks each.  SIDE 0: GemmArgs::r, 1: c.
//
// ALIGNED: every row of the operand starts at a 16-byte address and the rows'
// length (k in row form) is a multiple of 8, so each chunk is one 16-byte load
// straight into LDS; chunks past the ends get an offset past the buffer's
// range, which loads zeros.  Otherwise chunks pass through registers, and the
// ones that cross an end are read value by value.
template <int KS_, int ROWS, int NT, int SIDE, bool COL_, bool ALIGNED, bool PAIR>
struct Stage16 {
  static constexpr bool COL = COL_, DIRECT = ALIGNED;
  static constexpr int SCALED = 0;  // 4-bit weights: values per scale
  static constexpr int KS = KS_, CPR = KS / 8, CH = ROWS * CPR / NT;
  const uint16_t* p[2];  // the tile's first value, product 0; by segment, or gate and up for PAIR
  int64_t ld;
  int rows;  // rows of the operand from the tile's first (gate rows for PAIR)
  typedef std::conditional_t<ALIGNED, uint32_t, int64_t> Off;
  static constexpr Off OUTSIDE = ALIGNED ? (Off)0x80000000u : (Off)-1;
  Off off[CH];  // byte offset of each chunk from p, or OUTSIDE
  int at[CH];   // its first product (row form) or its product (column form)
  v4u reg[ALIGNED ? 1 : CH];

  __device__ __forceinline__ static int index(int j) { return (int)threadIdx.x + j * NT; }

  // `half` picks the operand where C has two halves; the operands of two
  // segments have one row stride.
  __device__ __forceinline__ void init(const GemmArgs& a, int half, int64_t r0) {
    const Operand* o = SIDE == 0 ? a.r + half : a.c;
    const int64_t all = SIDE == 0 ? a.rows : a.cols;
    ld = o->ld;
    p[0] = o->p + (COL ? r0 : r0 * ld);
    p[1] = PAIR || a.segments == 2 ? o[1].p + (COL ? r0 : r0 * ld) : p[0];
    rows = (int)(all - r0 < 0x7fffff00 ? all - r0 : 0x7fffff00);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = index(j);
      if constexpr (COL) {
        const int k = c / (ROWS / 8), r = ((c % (ROWS / 8)) ^ swz_col(k)) * 8;
        at[j] = k;
        off[j] = r < rows ? (Off)(k * ld + r) * 2 : OUTSIDE;
      } else {
        const int t = c / CPR, k = ((c % CPR) ^ swz_row<KS>(t)) * 8;
        const int r = weight_row<PAIR>(t);
        at[j] = k;
        off[j] = r < rows ? (Off)(r * ld + k) * 2 : OUTSIDE;
      }
    }
  }

  // A stage's loads: chunk(j) for j < CH, into (or on the way to) the stage at
  // lds, then next() to move on by KS products.  `left` products exist (all
  // further ones load as zeros; a DIRECT stage always issues CH loads).
  // Everything that moves is uniform over the block and is added to, not
  // computed anew: the scalar work of a step delays its matrix instructions.
  const uint16_t *from, *from2;
  int left;
  __device__ __forceinline__ void begin(int seg, int k0, int left_) {
    from = p[PAIR ? 0 : seg] + (COL ? k0 * ld : (int64_t)k0);
    from2 = PAIR ? p[1] + k0 : from;
    left = left_;
  }
  __device__ __forceinline__ void next() {
    const int64_t by = COL ? KS * ld : (int64_t)KS;
    from += by;
    if constexpr (PAIR) from2 += by;
    left -= KS;
  }
  __device__ __forceinline__ void chunk(lds_v4u* lds, int j) {
    if constexpr (ALIGNED) {
      const int w = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63) + j * NT;  // the wave's first chunk
      // a wave's 64 chunks are 8 or 16 rows, so all of them gate or all of them up
      const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)uniform(PAIR && ((w / CPR) & 32) ? from2 : from), (short)0,
                                                        0x7fffffff, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(lds + w), 16, at[j] < left ? off[j] : OUTSIDE, 0, 0, 0);
    } else {
      const int c = index(j);
      const uint16_t* q = PAIR && ((c / CPR) & 32) ? from2 : from;
      const int n = COL ? rows - ((c % (ROWS / 8)) ^ swz_col(c / (ROWS / 8))) * 8 : left - at[j];
      const bool in = off[j] != OUTSIDE && at[j] < left;
      reg[j] = load8_first(in ? (const uint16_t*)((const char*)q + off[j]) : q, in ? n : 0);
    }
  }
  // What chunk() left in registers, piece by piece.
  static constexpr int PIECES = ALIGNED ? 0 : CH;
  __device__ __forceinline__ void store(lds_v4u* lds, int j) { lds[index(j)] = reg[j]; }
};

// The tile of 4-bit weights, in row form: a thread takes 32 codes of one
// row (of one group) and writes them to LDS as scale * magnitude in the 16-bit
// type.  That is exact for scales of 6 significant bits, as q4_pack makes them:
// the magnitudes have 2.  In fp16 a row's scales are first multiplied by a power
// of two that takes the largest of them to [2^12, 2^13) (6 times as much is
// still below 65504), divided out of the sums again, and groups down to 2^-28 of
// that one are exact.  A scale whose products the type does not hold shows in
// `odd` as it passes.  The tile then gets a second pass over what the first has
// rounded away (bf16), or is summed anew by multiply_groups.  512 tokens, 4096 ->
// 16384 in bf16: 84 us for packed scales, 142 with one scale of 8 bits in the
// weight, 181 with nothing else; by multiply_groups alone 399 and 731.
template <class T, int ROWS, int NT, int GROUP, bool PAIR>
struct StageQ4 {
  static constexpr bool COL = false, DIRECT = false;
  static constexpr int SCALED = GROUP;
  static constexpr int KS = 64, CPR = KS / 8, CH = 1, W = KS / 16;  // 8 codes per word
  static_assert(ROWS * 2 == NT, "two threads per row");
  const uint8_t* p;
  const uint16_t* sp;
  float unit;
  int kp;
  bool in;
  bool rest;     // the second pass
  uint32_t odd;  // bit 0: it is needed; bit 1: it does not do
  v4u code;
  uint32_t sc;

  __device__ __forceinline__ void init(const GemmArgs& a, int, int64_t r0) {
    rest = false;
    odd = 0;
    const int t = threadIdx.x / 2, half = PAIR && (t & 32) ? 1 : 0;
    const int64_t row = r0 + weight_row<PAIR>(t);
    in = row < a.cols;
    kp = a.kp;
    p = a.codes[half] + (in ? row : 0) * (kp / 2);
    sp = a.scales[half] + (in ? row : 0) * (kp / GROUP);
    unit = a.unit[half] && in ? a.unit[half][row] : 1.0f;
  }
  int k, left;
  __device__ __forceinline__ void begin(int, int k0, int left_) {
    k = k0 + (threadIdx.x & 1) * (KS / 2);
    left = left_;
  }
  __device__ __forceinline__ void next() {
    k += KS;
    left -= KS;
  }
  __device__ __forceinline__ void chunk(lds_v4u*, int) {
    const bool on = in && k < kp && left > 0;
    code = on ? *(const v4u*)(p + k / 2) : v4u{};
    sc = on ? sp[k / GROUP] : 0u;
  }
  static constexpr int PIECES = W;
  __device__ __forceinline__ void store(lds_v4u* lds, int q) {
    const float s = BF16::up((uint16_t)sc) * unit;
    if (q == 0 && (sc & 0x7FFF) != 0 && (sc & 0x7F80) != 0x7F80) odd |= T::odd_e2m1(sc, unit);
    const int t = threadIdx.x / 2;
    const uint32_t c = code[q];
    lds_v4u* const to = lds + t * CPR + (((threadIdx.x & 1) * W + q) ^ swz_row<KS>(t));
    if constexpr (T::REST) {
      if (rest) {
        *to = v4u{T::template rest_e2m1<0>(c, s), T::template rest_e2m1<1>(c, s), T::template rest_e2m1<2>(c, s),
                  T::template rest_e2m1<3>(c, s)};
        return;
      }
    }
    *to = v4u{T::template scaled_e2m1<0>(c, s), T::template scaled_e2m1<1>(c, s), T::template scaled_e2m1<2>(c, s),
              T::template scaled_e2m1<3>(c, s)};
  }
};

// The 8 products [sub * 32 + (lane / 16) * 8, +8) of tile row r0 + lane % 16.
template <int KS, int ROWS, bool COL>
__device__ __forceinline__ v4u fragment(const lds_v4u* lds, int r0, int sub) {
  const int lane = threadIdx.x & 63;
  if constexpr (!COL) {
    const int r = r0 + (lane & 15);
    return lds[r * (KS / 8) + ((sub * 4 + (lane >> 4)) ^ swz_row<KS>(r))];
  } else {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s* lp;
    v2u h[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // 16 lanes read 4 LDS rows of 16 values and get them transposed: lane i
      // holds column i of the 4
      const int k = sub * 32 + (lane >> 4) * 8 + j * 4 + ((lane & 15) >> 2);
      const int c = r0 / 8 + ((lane & 3) >> 1);
      const lp at = (lp)(lds + k * (ROWS / 8) + (c ^ swz_col(k))) + (lane & 1);
      h[j] = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at));
    }
    return v4u{h[0][0], h[0][1], h[1][0], h[1][1]};
  }
}

// Four values of one row, columns c..c + 3 of `cols`, at any address that a value
// may have (global stores take it).
struct __attribute__((packed, aligned(2))) U64 {
  v2u v;
};
template <class T>
__device__ __forceinline__ void put4(void* out, int64_t row, int64_t c, int64_t cols, v4f v) {
  uint16_t* p = (uint16_t*)out + row + c;
  uint16_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = T::down(v[e]);
  if (c + 4 <= cols) {
    reinterpret_cast<U64*>(p)->v = v2u{b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < cols) p[e] = b[e];
  }
}

// A barrier before which at most N of the wave's loads into LDS may still be
// under way, and with STORES none of its LDS writes.  A fence would wait for
// every load, as they write LDS; fragments being read stay in flight: with 64
// products a stage none are (each has been used), with 32 the next stage's first
// ones, which is written again one barrier later.
template <int N, bool STORES>
__device__ __forceinline__ void stage_barrier() {
  static_assert(N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  if constexpr (STORES) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Results of row r, columns c..c + 3: bias, activation, rounding, store.
template <class T, int OUT, int ACT>
__device__ __forceinline__ void finish4(const GemmArgs& a, int half, int64_t r, int64_t c, v4f v[2]) {
  if constexpr (OUT == OUT_GATED) {
    if (a.pre) {
      float* g = a.pre + r * 2 * a.ld_pre + c;
      if (c + 4 <= a.cols) {
        *(v4f*)g = v[0];
        *(v4f*)(g + a.ld_pre) = v[1];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.cols) {
            g[e] = v[0][e];
            g[a.ld_pre + e] = v[1][e];
          }
      }
    }
    v4f h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = act_value<ACT>(v[0][e]) * v[1][e];
    put4<T>(a.out[0], r * a.ld_out, c, a.cols, h);
  } else {
    if (a.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < a.cols) v[0][e] += a.bias[c + e];
    }
    put4<T>(a.out[half], r * a.ld_out, c, a.cols, v[0]);
  }
}

// A block computes a BR x BC tile of C with waves of (BR / 2) x 64 each, from
// a ring of LDS stages.
//
// KS = 32: five stages.  While stage s is multiplied, stage s + 1 is complete,
// so its first fragments are read before the barrier between the two, and
// stages s + 2 .. s + 4 are on their way.
// KS = 64: two stages, one multiplied while the other is loaded.  For two
// operands in row form: their loads then take whole 128-byte lines.  Forward,
// two weights of 4096 -> 16384: 8192 tokens 1.87 ms against 1.98 with 32, 1021
// tokens of 1000 -> 2731 28 us against 35.  Operands in column form gain from
// the deeper ring: gx at 8192 tokens 1.81 ms against 2.16 with 64.
template <int KS>
constexpr int STAGES = KS == 32 ? 5 : 2;

template <class SR, class SC>
__device__ __forceinline__ void load_chunk(SR& sr, SC& sc, lds_v4u* tr, lds_v4u* tc, int i) {
  if (i < SR::CH) sr.chunk(tr, i);
  else sc.chunk(tc, i - SR::CH);
}

template <class SR, class SC>
__device__ __forceinline__ void store_piece(SR& sr, SC& sc, lds_v4u* tr, lds_v4u* tc, int i) {
  if constexpr (SR::PIECES > 0) {
    if (i < SR::PIECES) sr.store(tr, i);
  }
  if constexpr (SC::PIECES > 0) {
    if (i >= SR::PIECES) sc.store(tc, i - SR::PIECES);
  }
}
// The loads of an operand that goes straight into LDS, or of one that does not.
template <bool DIRECT, class S>
__device__ __forceinline__ void load_if(S& s, lds_v4u* to) {
  if constexpr (S::DIRECT == DIRECT) {
#pragma unroll
    for (int j = 0; j < S::CH; ++j) s.chunk(to, j);
  }
}

// The order of a stage's LDS reads, matrix instructions and loads: groups of 4
// instructions that share a row fragment, each with a share of the reads
// before it and of the loads after it.  Left alone, the compiler reads each
// fragment right before its use and issues all loads at once, and the wave
// waits out the LDS latency and the issue of the loads.
template <int READS, int LOADS>
__device__ __forceinline__ void group_order() {
  constexpr int MFMA = 0x8, VMEM = 0x10, DS_READ = 0x100;
  if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(DS_READ, READS, 0);
  __builtin_amdgcn_sched_group_barrier(MFMA, 4, 0);
  if constexpr (LOADS > 0) __builtin_amdgcn_sched_group_barrier(VMEM, LOADS, 0);
}

// KS = 32: the products of stage `now`, with the reads of the next one's first
// fragments from `then` and the loads into `to` between them.  The three are
// distinct, which the compiler has to know (__restrict__): it makes reads wait
// for loads into LDS that they might alias.
constexpr int EARLY = 3;  // row fragments read a stage ahead, beside the column fragments
template <class T, int BR, int BC, int P, class SR, class SC, int NR>
__device__ __forceinline__ void multiply32(v4f (&acc)[4][NR], v4u (&fc)[2][4], v4u (&fr)[2][EARLY], SR& sr, SC& sc,
                                           int wr, int wc, const lds_v4u* __restrict__ now,
                                           const lds_v4u* __restrict__ then, lds_v4u* __restrict__ to) {
  constexpr int LR = BR * SR::CPR, MID = NR - EARLY, READS = NR + 4, CHUNKS = SR::CH + SC::CH;
  v4u f[NR];
#pragma unroll
  for (int i = 0; i < EARLY; ++i) f[i] = fr[P][i];
  Unroll<0, NR>::run([&](auto g) {
    constexpr int G = decltype(g)::value;
    constexpr int R0 = READS * G / NR, R1 = READS * (G + 1) / NR, L0 = CHUNKS * G / NR, L1 = CHUNKS * (G + 1) / NR;
    Unroll<R0, R1>::run([&](auto r) {
      constexpr int R = decltype(r)::value;
      if constexpr (R < MID) f[R + EARLY] = fragment<32, BR, SR::COL>(now, wr + (R + EARLY) * 16, 0);
      else if constexpr (R < MID + 4) fc[P ^ 1][R - MID] = fragment<32, BC, SC::COL>(then + LR, wc + (R - MID) * 16, 0);
      else fr[P ^ 1][R - MID - 4] = fragment<32, BR, SR::COL>(then, wr + (R - MID - 4) * 16, 0);
    });
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i][G] = T::mfma(fc[P][i], f[G], acc[i][G]);
    Unroll<L0, L1>::run([&](auto l) { load_chunk(sr, sc, to, to + LR, decltype(l)::value); });
    auto instructions = [](int n) constexpr {  // LDS reads of the first n fragments
      const int c = n < MID ? 0 : n < MID + 4 ? n - MID : 4;
      return (n - c) * (SR::COL ? 2 : 1) + c * (SC::COL ? 2 : 1);
    };
    group_order<instructions(R1) - instructions(R0), L1 - L0>();
  });
}

// KS = 64: the products of stage `now`.  The first fragments are read ahead,
// the others spread over the first two thirds of the groups; the loads into
// tr and tc, the next stage's two parts, come within the first quarter (spread
// over half of the groups they end late for the barrier: forward at 8192 tokens
// 2.30 ms, not 2.21).  An operand that passes through registers is loaded first
// and stored last.
template <class T, int BR, int BC, class SR, class SC, int NR>
__device__ __forceinline__ void multiply64(v4f (&acc)[4][NR], SR& sr, SC& sc, int wr, int wc,
                                           const lds_v4u* __restrict__ now, lds_v4u* __restrict__ tr,
                                           lds_v4u* __restrict__ tc) {
  constexpr int LR = BR * SR::CPR, GROUPS = 2 * NR, HALF = 4 + NR, READS = 2 * HALF, FIRST = 4 + 3;
  constexpr int LOADS = (SR::DIRECT ? SR::CH : 0) + (SC::DIRECT ? SC::CH : 0), PIECES = SR::PIECES + SC::PIECES;
  v4u f[2][NR], fc[2][4];
  load_if<false>(sr, tr);
  load_if<false>(sc, tc);
  Unroll<0, GROUPS>::run([&](auto g) {
    constexpr int G = decltype(g)::value;
    // fragments read before group n, in the order fc then fr, half after half
    auto before = [](int n) constexpr {
      const int c = FIRST + ((READS - FIRST) * n * 3 + 2 * GROUPS - 1) / (2 * GROUPS);
      return n < 0 ? 0 : c < READS ? c : READS;
    };
    constexpr int R0 = before(G - 1), R1 = before(G);
    constexpr int LA = 4 * LOADS * G / GROUPS, LB = 4 * LOADS * (G + 1) / GROUPS;
    constexpr int L0 = LA < LOADS ? LA : LOADS, L1 = LB < LOADS ? LB : LOADS;
    Unroll<R0, R1>::run([&](auto r) {
      constexpr int R = decltype(r)::value, H = R / HALF, I = R % HALF;
      if constexpr (I < 4) fc[H][I] = fragment<64, BC, SC::COL>(now + LR, wc + I * 16, H);
      else f[H][I - 4] = fragment<64, BR, SR::COL>(now, wr + (I - 4) * 16, H);
    });
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i][G % NR] = T::mfma(fc[G / NR][i], f[G / NR][G % NR], acc[i][G % NR]);
    Unroll<L0, L1>::run([&](auto l) {
      load_chunk(sr, sc, tr, tc, decltype(l)::value + (SR::DIRECT ? 0 : SR::CH));
    });
    group_order<R1 - R0, L1 - L0>();
  });
#pragma unroll
  for (int i = 0; i < PIECES; ++i) store_piece(sr, sc, tr, tc, i);
}

// The two low bits of all lanes of the block, or-ed.  LDS is free for it, before and after.
template <int WAVES>
__device__ __forceinline__ uint32_t or_lanes(uint32_t bits, lds_v4u* lds) {
  const uint32_t mine = (__ballot(bits & 1) != 0 ? 1u : 0u) | (__ballot(bits & 2) != 0 ? 2u : 0u);
  __syncthreads();
  lds[threadIdx.x / 64] = v4u{mine, 0, 0, 0};
  __syncthreads();
  uint32_t all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all |= lds[w][0];
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(all);
}

// The sums over products [from, to) of 16 columns (of gate and up, H = 2) and
// all of a wave's rows, for 4-bit weights of any scales: 32 products of the bare
// magnitudes at a time, times the scale in fp32.  r, w: the first row of x and
// of the weights.  Operands come from global memory as they are needed: weights
// that take this path are right, not fast.
template <class T, int GROUP, int H, bool WHOLE, int NR>
__device__ __forceinline__ void multiply_groups(v4f (&sums)[H][NR], const GemmArgs& a, int64_t r, int64_t w, int from,
                                                int to) {
  const int lane = threadIdx.x & 63, o = lane >> 4;
  // rows past the ends: the last one, whose results there go nowhere
  auto row = [&](int64_t first, int n) { return first + (lane & 15) < n ? first + (lane & 15) : (int64_t)n - 1; };
  const int64_t wr = row(w, a.cols);
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int j = 0; j < NR; ++j) sums[h][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = from; k0 < to; k0 += 32) {
    const int k = k0 + o * 8;
    v4u fc[H];
    v4f s[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const uint32_t c = *(const uint32_t*)(a.codes[h] + wr * (a.kp / 2) + k / 2);
      const float scale = BF16::up(a.scales[h][wr * (a.kp / GROUP) + k0 / GROUP]);
      fc[h] = v4u{T::template from_e2m1<0>(c), T::template from_e2m1<1>(c), T::template from_e2m1<2>(c),
                  T::template from_e2m1<3>(c)};
#pragma unroll
      for (int e = 0; e < 4; ++e) s[h][e] = __shfl(scale, o * 4 + e);
    }
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      const uint16_t* x = a.r[0].p + row(r + j * 16, a.rows) * a.r[0].ld;
      v4u f;
      if constexpr (WHOLE) {
        f = load8(x + (k < a.k ? k : 0));
        f = k < a.k ? f : v4u{0, 0, 0, 0};
      } else {
        f = load8_first(x + k, a.k - k);
      }
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const v4f sum = T::mfma(fc[h], f, v4f{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[h][j][e] = fmaf(s[h][e], sum[e], sums[h][j][e]);
      }
    }
  }
}

// A tile of C: its row and column, rows numbered over both halves.
struct TileAt {
  uint32_t r, c;
};
// Tile number t of rows x cols tiles: 8 tile rows at a time, column after column.
__device__ __forceinline__ TileAt tile_number(uint32_t t, uint32_t rows, uint32_t cols) {
  const uint32_t group = 8 * cols, first = t / group * 8, some = rows - first < 8 ? rows - first : 8;
  return {first + t % group % some, t % group / some};
}
// Workgroups go to the 8 dies in turn; each die gets a run of the `all` tiles, which
// share operands in its L2.
__device__ __forceinline__ uint32_t die_tile(uint32_t id, uint32_t all) {
  const uint32_t die = id & 7;
  return die * (all / 8) + (die < all % 8 ? die : all % 8) + id / 8;
}
__device__ __forceinline__ TileAt tile_at(uint32_t id, uint32_t rows, uint32_t cols) {
  return tile_number(die_tile(id, rows * cols), rows, cols);
}

// The products of part `part` of a.parts of one tile.
template <class T, class SR, class SC, int OUT, int BR, int BC>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, lds_v4u* const lds, const TileAt at, uint32_t part) {
  constexpr int KS = SR::KS, NR = BR / 32, PAIR = OUT == OUT_GATED;
  constexpr int LR = BR * SR::CPR, LC = BC * SR::CPR, STAGE = LR + LC, CHUNKS = SR::CH + SC::CH;
  constexpr int LOADS = (SR::DIRECT ? SR::CH : 0) + (SC::DIRECT ? SC::CH : 0);  // into LDS, per stage and thread
  constexpr bool REGS = !SR::DIRECT || !SC::DIRECT;                             // some pass through registers
  const int half = at.r >= (uint32_t)a.tiles_r;
  const int64_t r0 = (int64_t)(at.r - half * a.tiles_r) * BR;
  const int64_t c0 = (int64_t)at.c * (PAIR ? BC / 2 : BC);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int wr = (wave & 1) * (BR / 2), wc = (wave >> 1) * 64;
  v4f acc[4][NR];  // [column group][row group]: lane holds row lane % 16, columns (lane / 16) * 4 + 0..3
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NR; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  SR sr;
  SC sc;
  const int steps = ceil_div(a.k, KS), total = steps * a.segments;
  const int begin = (int)((int64_t)total * part / a.parts), end = (int)((int64_t)total * (part + 1) / a.parts);
  sr.init(a, half, r0);
  sc.init(a, 0, c0);
  // Before the loads of step s: they start, change operands or end there.
  int until = begin < steps && end > steps ? steps : end;
  auto restart = [&] {
    const int seg = begin >= steps ? 1 : 0, k0 = (begin - seg * steps) * KS;
    sr.begin(seg, k0, begin < end ? a.k - k0 : 0);
    sc.begin(seg, k0, begin < end ? a.k - k0 : 0);
  };
  restart();
  auto start = [&](int s) {
    if (s != until) return;
    const bool more = s < end;
    sr.begin(1, 0, more ? a.k : 0);
    sc.begin(1, 0, more ? a.k : 0);
    until = more ? end : -1;
  };
  auto next = [&] {
    sr.next();
    sc.next();
  };
  auto load = [&](lds_v4u* to) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) load_chunk(sr, sc, to, to + LR, j);
    next();
  };
  auto store = [&](lds_v4u* to) {
#pragma unroll
    for (int i = 0; i < SR::PIECES + SC::PIECES; ++i) store_piece(sr, sc, to, to + LR, i);
  };
  [[maybe_unused]] uint32_t odd = 0;
  if constexpr (KS == 64) {
    static_assert(!SR::COL && !SC::COL, "one segment");
    auto pass = [&] {
      load(lds);
      store(lds);
      for (int s = begin; s < end; ++s) {
        const int b = (s - begin) & 1;
        stage_barrier<0, REGS>();
        multiply64<T, BR, BC>(acc, sr, sc, wr, wc, lds + b * STAGE, lds + (b ^ 1) * STAGE,
                              lds + (b ^ 1) * STAGE + LR);
        next();
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load may reach LDS after what uses it next
    };
    if constexpr (SC::SCALED == 0) {
      pass();
    } else {
      for (;;) {
        pass();
        if (T::REST && sc.rest) break;
        odd = or_lanes<BC / 32>(sc.odd, lds);
        if (!T::REST || odd != 1) break;
        // an infinite sum stays: the second pass would add infinity times zero
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) z += acc[i][j][e] * 0.0f;
        odd |= or_lanes<BC / 32>(z == 0.0f ? 0 : 2, lds);
        if (odd & 2) break;
        sc.rest = true;
        restart();
      }
    }
  } else {
    // Stages loaded straight into LDS are 4 steps ahead.  Those that pass
    // through registers are in LDS two steps ahead and in registers three;
    // with one operand of each kind both are.
    constexpr int AHEAD = REGS ? 3 : STAGES<KS> - 1;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      start(begin + i);
      load(lds + i * STAGE);
      if (REGS && i < AHEAD - 1) store(lds + i * STAGE);
    }
    stage_barrier<(AHEAD - 1) * LOADS, REGS>();
    v4u fc[2][4], fr[2][EARLY];
#pragma unroll
    for (int i = 0; i < 4; ++i) fc[0][i] = fragment<KS, BC, SC::COL>(lds + LR, wc + i * 16, 0);
#pragma unroll
    for (int i = 0; i < EARLY; ++i) fr[0][i] = fragment<KS, BR, SR::COL>(lds, wr + i * 16, 0);
    int cur = 0;  // the stage being multiplied
    auto step = [&](auto phase, int s) {
      constexpr int P = decltype(phase)::value;
      auto stage = [&](int d) { return lds + (cur + d < STAGES<KS> ? cur + d : cur + d - STAGES<KS>) * STAGE; };
      stage_barrier<(AHEAD - 2) * LOADS, REGS>();
      if constexpr (REGS) store(stage(AHEAD - 1));
      start(s + AHEAD);
      multiply32<T, BR, BC, P>(acc, fc, fr, sr, sc, wr, wc, stage(0), stage(1), stage(AHEAD));
      next();
      cur = cur + 1 < STAGES<KS> ? cur + 1 : 0;
    };
    for (int s = begin; s < end; s += 2) {
      step(std::integral_constant<int, 0>{}, s);
      if (s + 1 < end) step(std::integral_constant<int, 1>{}, s + 1);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load may reach LDS after the block has left it
  constexpr int H = PAIR ? 2 : 1;
  const int64_t c1 = c0 + (PAIR ? wc / 2 : wc) + (lane >> 4) * 4;
  // The sums of row group j and column group i.
  auto put = [&](auto act, int i, int j, v4f v[2]) {
    const int64_t r = r0 + wr + j * 16 + (lane & 15), c = c1 + i * 16;
    if (r >= a.rows || c >= a.cols) return;
    if (a.part) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int64_t plane = (int64_t)part * (PAIR ? 2 : a.halves) + (PAIR ? h : half);
        *(v4f*)(a.part + (plane * a.part_rows + r) * a.ld_part + c) = v[h];
      }
    } else {
      finish4<T, OUT, decltype(act)::value>(a, half, r, c, v);
    }
  };
  auto finish = [&](auto act) {
    // Row by row, so that the two halves of a 128-byte line are written one
    // after the other.
    v4f back[4 / H][H];  // what the 4-bit weights' rows were divided by
#pragma unroll
    for (int i = 0; i < 4 / H; ++i)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t c = c1 + i * 16 + e;
          back[i][h][e] = a.unit[h] && c < a.cols ? 1.0f / a.unit[h][c] : 1.0f;
        }
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
      for (int i = 0; i < 4 / H; ++i) {
        v4f v[2] = {acc[i][j] * back[i][0], v4f{}};
        if constexpr (PAIR) v[1] = acc[i + 2][j] * back[i][H - 1];
        put(act, i, j, v);
      }
  };
  if constexpr (PAIR)
    with_act(a.act, finish);
  else
    finish(std::integral_constant<int, 0>{});
  // Each lane stores over what it has stored: the sums above need no registers then.
  if constexpr (SC::SCALED != 0) {
    if (odd & 2) {
#pragma unroll 1
      for (int i = 0; i < 4 / H; ++i) {
        v4f sums[H][NR];
        multiply_groups<T, SC::SCALED, H, SR::DIRECT>(sums, a, r0 + wr, c0 + (PAIR ? wc / 2 : wc) + i * 16, begin * KS,
                                                      end < steps ? end * KS : a.k);
        with_act(PAIR ? a.act : 0, [&](auto act) {
#pragma unroll
          for (int j = 0; j < NR; ++j) {
            v4f v[2] = {sums[0][j], sums[H - 1][j]};
            put(act, i, j, v);
          }
        });
      }
    }
  }
}

template <class T, class SR, class SC, int OUT, int BR, int BC>
__global__ __launch_bounds__(BC / 64 * 128) void dense_gemm_kernel(GemmArgs a) {
  static_assert(SR::KS == SC::KS, "one ring");
  [[maybe_unused]] __shared__ v4u lds[STAGES<SR::KS> * (BR + BC) * SR::CPR];
#ifdef __HIP_DEVICE_COMPILE__  // the host has no LDS pointers
  const uint32_t rows = a.tiles_r * a.halves, all = rows * a.tiles_c;
  gemm_tile<T, SR, SC, OUT, BR, BC>(a, (lds_v4u*)lds, tile_at(blockIdx.x % all, rows, a.tiles_c), blockIdx.x / all);
#endif
}

// Joins the parts of a split product: four columns of one row per thread.
template <class T, int OUT, int ACT>
__device__ __forceinline__ void join(const GemmArgs& a) {
  constexpr int H = OUT == OUT_GATED ? 2 : 1;
  const int q = a.ld_part / 4;
  const int64_t n = (int64_t)a.rows * q * (OUT == OUT_GATED ? 1 : a.halves);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / q;  // of both halves
    const int half = row >= a.rows;
    const int64_t c = i % q * 4;
    const int64_t plane = (int64_t)a.part_rows * a.ld_part, step = plane * (OUT == OUT_GATED ? 2 : a.halves);
    v4f v[2] = {};
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float* p = a.part + h * plane + row * a.ld_part + c;
      v4f s = *(const v4f*)p;
#pragma unroll 8
      for (int k = 1; k < a.parts; ++k) s += *(const v4f*)(p + k * step);
      v[h] = s;
    }
    finish4<T, OUT, ACT>(a, half, row - half * (int64_t)a.rows, c, v);
  }
}
template <class T, int OUT>
__global__ __launch_bounds__(256) void dense_join_kernel(GemmArgs a) {
  with_act(OUT == OUT_GATED ? a.act : 0, [&](auto act) { join<T, OUT, decltype(act)::value>(a); });
}

// Every row of the operand starts at a 16-byte address, and a tile's offsets
// stay below 2^31 bytes.
inline bool aligned_rows(const Operand& o) {
  return ((uintptr_t)o.p & 15) == 0 && o.ld % 8 == 0 && o.ld < (1 << 21);
}

// Operands whose rows do not start at 16-byte addresses, or end inside 16
// bytes, are copied once into rows that do (ld = k rounded up to 8, zeros past
// k): a tile's loads then go straight into LDS.  The copies cost 2 bytes each
// way per value; the products through registers, which operands with other
// addresses alone still take, run at half of the rate in the forward and a fifth
// in column form: training step at 4000 tokens, 2047 -> 4001: 544 us against 1702.
struct Realign {
  const uint16_t* p[3];
  int64_t ld[3];
  int64_t rows[3];  // 0: none
  uint16_t* out[3];
  int k, kp;
};
static __global__ __launch_bounds__(256) void dense_realign_kernel(Realign a) {
  const int per = a.kp / 8;
#pragma unroll
  for (int o = 0; o < 3; ++o) {
    const int64_t n = a.rows[o] * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
      const int64_t row = i / per;
      const int c = (int)(i % per) * 8;
      *(v4u*)(a.out[o] + i * 8) = load8_first(a.p[o] + row * a.ld[o] + c, a.k - c);
    }
  }
}

// Whether sizes and strides ask for copies, and their rows' length.
inline bool realigns(int k, int64_t ld_a, int64_t ld_b) {
  return (k % 8 || ld_a % 8 || ld_b % 8) && round_up(k, 8) < (1 << 21);
}
inline size_t realign_bytes(int64_t rows, int k) { return (size_t)round_up(rows * round_up(k, 8) * 2, 16); }

// Collects the operands that need a copy; each gets `rows` rows at *ws.
struct Realigner {
  Realign a = {};
  int n = 0;
  char* ws;
  Realigner(int k, void* ws_) : ws((char*)ws_) {
    a.k = k;
    a.kp = (int)round_up(k, 8);
  }
  bool fits(const Operand& o) const { return aligned_rows(o) && a.k % 8 == 0; }
  // Two operands that share a row stride are copied together or not at all.
  void add_pair(Operand& o, Operand& q, int64_t rows) {
    if (fits(o) && fits(q)) return;
    o = copy(o, rows);
    q = copy(q, rows);
  }
  void add(Operand& o, int64_t rows) {
    if (!fits(o)) o = copy(o, rows);
  }
  Operand copy(const Operand& o, int64_t rows) {
    a.p[n] = o.p;
    a.ld[n] = o.ld;
    a.rows[n] = rows;
    a.out[n] = (uint16_t*)ws;
    ws += realign_bytes(rows, a.k);
    return {a.out[n++], a.kp};
  }
  int run(hipStream_t s) {
    int64_t most = 0;
    for (int i = 0; i < n; ++i)
      if (a.rows[i] > most) most = a.rows[i];
    const int64_t units = most * (a.kp / 8);
    if (units == 0) return QCONV_OK;
    dense_realign_kernel<<<(unsigned)(units < (1 << 20) ? (units + 255) / 256 : 4096), 256, 0, s>>>(a);
    return hip_status();
  }
};

struct GemmPlan {
  int tile;  // rows and columns of a block's tile
  int parts;
  size_t bytes;  // of GemmArgs::part
};

// Tiles of 256 x 256 where they fill the 256 compute units by themselves, else
// 128 x 128, two blocks per unit.  Few tiles: their products are split over
// blocks until there are about 256, as long as each keeps 512 products (gx of
// 512 tokens, 4096 -> 1024: 35 us in 8 parts, 116 in one, 36 in 16).  With
// `long_sums` (gx, whose sums run over both halves of 2f) also the larger
// tiles are split if each part keeps 2048 products: gx of 4096 tokens, 8192 ->
// 2048: 128 tiles in two parts 215 us, 512 small tiles 313; of 256 tokens,
// 1024 -> 8192, with 512 products each: 37 us against 32.
inline GemmPlan gemm_plan(int64_t rows, int64_t cols, int64_t products, int halves, bool gated, bool aligned,
                          bool long_sums) {
  const int planes = gated ? 2 : halves;
  auto tiles = [&](int b) {
    const int64_t across = gated ? b / 2 : b;
    const int64_t n = (rows + b - 1) / b * ((cols + across - 1) / across) * halves;
    return n > 0 ? n : 1;
  };
  auto split = [&](int tile, int64_t parts) {
    return GemmPlan{tile, (int)parts, parts > 1 ? (size_t)parts * planes * rows * round_up(cols, 4) * 4 : 0};
  };
  const int64_t big = tiles(256), small = tiles(128);
  if (aligned && big >= 256) return split(256, 1);
  if (aligned && long_sums && 256 / big * big >= 192 && products / (256 / big) >= 2048) return split(256, 256 / big);
  int64_t parts = small >= 192 ? 1 : 256 / small;
  if (parts > products / 512) parts = products / 512;
  return split(128, parts < 1 ? 1 : parts);
}

template <class T, class SR, class SC, int OUT, int B>
int run_gemm_tiles(GemmArgs& a, hipStream_t s) {
  a.tiles_r = ceil_div(a.rows, B);
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? B / 2 : B);
  const int64_t blocks = (int64_t)a.tiles_r * a.tiles_c * a.halves * a.parts;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  if (a.parts == 1) a.part = nullptr;
  a.part_rows = a.rows;
  a.ld_part = (int)round_up(a.cols, 4);
  dense_gemm_kernel<T, SR, SC, OUT, B, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a);
  if (a.parts > 1) {
    const int64_t n = (int64_t)a.rows * (a.ld_part / 4) * (OUT == OUT_GATED ? 1 : a.halves);
    dense_join_kernel<T, OUT><<<(unsigned)(n < (1 << 20) ? (n + 255) / 256 : 4096), 256, 0, s>>>(a);
  }
  return hip_status();
}

}  // namespace qc
