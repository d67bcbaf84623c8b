// moe_gemm.hip -- the experts' products: rows offsets[e] .. offsets[e + 1] of x
// with the weights of expert e, forward and backward, in 16-bit types.
//   gated    h = act(x Wg_e^T) (x Wu_e^T), as ffn.hip for each expert's rows
//   linear   y = x W_e^T;  gx = gy W_e;  gW_e = gy_e^T x_e
// One launch per product for all experts, on the tiles of dense_gemm.h: a block
// finds its expert and rows from the offsets, which stay on the device.
//
// Bound by the matrix cores at many rows, by reading the weights at few.  Measured in
// bf16, 16384 rows of 8 experts (half of them one expert's), 2048 <-> 4096, 0.55 TFLOP
// each: forward 652 us with the 0.54 GB of pre (509 without), gx 495, both weight
// gradients 532 (840 to 1110 TFLOP/s); 8192 rows of 16 experts, 2048 -> 2048, linear:
// forward 101, gx 102, weight gradients 115 (600 to 680).  What is lost against one
// weight's products: tiles that an expert's last rows do not fill, the tail of the
// last tiles, and sums too short to hide a tile's start and end.
#include "dense_ffn.h"
#include "dense_rows.h"
#include "moe.h"
#include "moe_groups.h"

#include "qconv_internal.h"

namespace qc {

namespace {

// The arguments of one expert's rows.
template <int OUT>
__device__ __forceinline__ void take_rows(GemmArgs& a, const GroupRows& rows) {
  const int64_t first = __builtin_amdgcn_readfirstlane(rows.first);
#pragma unroll
  for (int i = 0; i < 2; ++i) a.r[i].p += first * a.r[i].ld;
  a.rows = __builtin_amdgcn_readfirstlane(rows.count);
  a.out[0] = (uint16_t*)a.out[0] + first * a.ld_out;
  if (OUT == OUT_GATED && a.pre) a.pre += first * 2 * a.ld_pre;
}

// Tiles of 256 x 256, one block of which fits a compute unit: as many as fill the
// chip's 256 units a whole number of times are taken whole, the others' products are
// split over the units that would be idle and joined by moe_tail_kernel (gx of 16384
// rows of 8 experts, 4096 -> 2048: about 544 tiles, 500 us where three whole rounds
// take 620; forward of 8192 rows of 16, 2048 -> 2048: 108 and 122).
struct Tail {
  uint32_t full, rest;  // tiles
  int parts;            // of each of the rest
};
constexpr int TAIL_TILE = 256 * 256;  // fp32 sums of a part
__device__ __forceinline__ Tail tail_of(uint32_t all, int64_t products) {
  Tail t;
  t.full = all & ~255u;
  t.rest = all - t.full;
  int64_t parts = t.rest ? 256 / t.rest : 1;
  if (parts > products / 512) parts = products / 512;
  t.parts = parts > 16 ? 16 : parts > 1 ? (int)parts : 1;
  return t;
}

// The products whose rows are the batch's (forward, gx).
template <class T, class SR, class SC, int OUT, int B>
__global__ __launch_bounds__(B / 64 * 128) void moe_gemm_kernel(GemmArgs a, Groups g, int64_t step_c) {
  [[maybe_unused]] __shared__ v4u lds[STAGES<SR::KS> * (B + B) * SR::CPR];
#ifdef __HIP_DEVICE_COMPILE__  // the host has no LDS pointers
  const GroupPieces pieces(g, B);
  const uint32_t all = (uint32_t)pieces.total * a.tiles_c;
  uint32_t part, tile;
  [[maybe_unused]] float* sums = nullptr;
  if constexpr (B == 256) {
    const Tail tail = tail_of(all, (int64_t)a.k * a.segments);
    part = 0;
    if (blockIdx.x < tail.full) {
      tile = die_tile(blockIdx.x, tail.full);
      a.parts = 1;
    } else {
      const uint32_t i = (blockIdx.x - tail.full) / tail.parts;
      if (i >= tail.rest) return;
      tile = tail.full + i;
      a.parts = tail.parts;
      part = (blockIdx.x - tail.full) % tail.parts;
      if (tail.parts > 1) sums = a.part + (int64_t)i * tail.parts * TAIL_TILE;
    }
  } else {
    // the parts of one tile lie as many blocks apart as are launched for each
    const uint32_t blocks = gridDim.x / a.parts, id = blockIdx.x % blocks;
    part = blockIdx.x / blocks;
    if (id >= all) return;
    tile = die_tile(id, all);
  }
  TileAt at = tile_number(tile, pieces.total, a.tiles_c);
  int e, piece;
  pieces.find(g, at.r, e, piece);
  const GroupRows rows = group_rows(g, e);
  take_rows<OUT>(a, rows);
#pragma unroll
  for (int i = 0; i < 2; ++i) a.c[i].p += e * step_c;
  at.r = piece;
  if constexpr (B == 256) {
    a.part = sums;
    if (sums) {  // [parts][2 if gated][256][columns of a tile]
      a.part_rows = 256;
      a.ld_part = OUT == OUT_GATED ? 128 : 256;
      a.part -= ((int64_t)at.r * 256 + at.c) * a.ld_part;
    }
  } else if (a.part) {
    a.part += (int64_t)rows.first * a.ld_part;
  }
  a.tiles_r = 0x7fffffff;  // one half
  gemm_tile<T, SR, SC, OUT, B, B>(a, (lds_v4u*)lds, at, part);
#endif
}

// Joins the tiles that moe_gemm_kernel has split: 16 blocks a tile.
template <class T, int OUT>
__global__ __launch_bounds__(256) void moe_tail_kernel(GemmArgs a, Groups g) {
  constexpr int H = OUT == OUT_GATED ? 2 : 1, COLS = 256 / H;
  const GroupPieces pieces(g, 256);
  const Tail tail = tail_of((uint32_t)pieces.total * a.tiles_c, (int64_t)a.k * a.segments);
  const uint32_t i = blockIdx.x / 16;
  if (i >= tail.rest || tail.parts == 1) return;
  const TileAt at = tile_number(tail.full + i, pieces.total, a.tiles_c);
  int e, piece;
  pieces.find(g, at.r, e, piece);
  take_rows<OUT>(a, group_rows(g, e));
  const float* sums = a.part + (int64_t)i * tail.parts * TAIL_TILE;
  with_act(OUT == OUT_GATED ? a.act : 0, [&](auto act) {
    for (int q = threadIdx.x; q < 16 * COLS / 4; q += 256) {
      const int row = blockIdx.x % 16 * 16 + q / (COLS / 4), col = q % (COLS / 4) * 4;
      const int64_t r = (int64_t)piece * 256 + row, c = (int64_t)at.c * COLS + col;
      if (r >= a.rows || c >= a.cols) continue;
      v4f v[2] = {};
#pragma unroll
      for (int h = 0; h < H; ++h)
        for (int p = 0; p < tail.parts; ++p)
          v[h] += *(const v4f*)(sums + ((int64_t)(p * H + h) * 256 + row) * COLS + col);
      finish4<T, OUT, decltype(act)::value>(a, 0, r, c, v);
    }
  });
}

// The join of split products, for the rows that groups have.
template <class T, int OUT>
__global__ __launch_bounds__(256) void moe_join_kernel(GemmArgs a, Groups g) {
  const int first = g.offsets[0] < 0 ? 0 : g.offsets[0], end = g.offsets[g.n] < g.rows ? g.offsets[g.n] : g.rows;
  a.rows = end - first;
  a.part += (int64_t)first * a.ld_part;
  a.out[0] = (uint16_t*)a.out[0] + first * a.ld_out;
  if (OUT == OUT_GATED && a.pre) a.pre += (int64_t)first * 2 * a.ld_pre;
  with_act(OUT == OUT_GATED ? a.act : 0, [&](auto act) { join<T, OUT, decltype(act)::value>(a); });
}

// The products over the batch's rows (weight gradients): a.rows and a.cols are
// the weight's.  An expert's rows are taken `size` at a time, so that experts of
// unequal share, or few of them, fill the chip; sums of an expert with several such
// pieces go to a.part.
template <class T, class SR, class SC, int B>
__global__ __launch_bounds__(B / 64 * 128) void moe_gemm_w_kernel(GemmArgs a, Groups g, int size, int uncut, int64_t step_out) {
  [[maybe_unused]] __shared__ v4u lds[STAGES<SR::KS> * (B + B) * SR::CPR];
#ifdef __HIP_DEVICE_COMPILE__
  // one piece after the other, each over all dies: their sums differ in length
  const uint32_t per = a.tiles_r * a.halves, all = per * a.tiles_c;
  size = group_size(g, size, uncut);
  const GroupPieces pieces(g, size, true);
  const int p = blockIdx.x / all;
  if (p >= pieces.total) return;
  const TileAt at = tile_at(blockIdx.x % all, per, a.tiles_c);
  int e, piece = 0;
  // the longest sums first: the chip is then busy to the end
  if (g.n <= 64 && pieces.total == g.n) e = group_by_size(g, p);
  else pieces.find(g, p, e, piece);
  const GroupRows rows = group_rows(g, e);
  const int64_t begin = (int64_t)piece * size, first = __builtin_amdgcn_readfirstlane(rows.first) + begin;
  const int count = __builtin_amdgcn_readfirstlane(rows.count);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a.r[i].p += first * a.r[i].ld;
    a.out[i] = (uint16_t*)a.out[i] + e * step_out;
  }
  a.c[0].p += first * a.c[0].ld;
  a.k = count - begin < size ? count - (int)begin : size;
  a.part = count > size ? a.part + group_part(first - begin, piece, size) * a.halves * a.part_rows * a.ld_part : nullptr;
  gemm_tile<T, SR, SC, OUT_PLAIN, B, B>(a, (lds_v4u*)lds, at, 0);
#endif
}

// The join of the experts' pieces: blockIdx.y counts the experts with several.
template <class T>
__global__ __launch_bounds__(256) void moe_join_w_kernel(GemmArgs a, Groups g, int size, int uncut, int64_t step_out) {
  size = group_size(g, size, uncut);
  const GroupPieces several(g, size, false, true);
  if ((int)blockIdx.y >= several.total) return;
  int e, unused;
  several.find(g, blockIdx.y, e, unused);
  const GroupRows rows = group_rows(g, e);
  const int n = (rows.count - 1) / size + 1, q = a.ld_part / 4;
  const int64_t plane = (int64_t)a.part_rows * a.ld_part;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)a.halves * a.part_rows * q; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / q;  // of both halves
    const int half = row >= a.part_rows, c = (int)(i % q) * 4;
    v4f v[2] = {};
#pragma unroll 4
    for (int p = 0; p < n; ++p)
      v[0] += *(const v4f*)(a.part + group_part(rows.first, p, size) * a.halves * plane + row * a.ld_part + c);
    GemmArgs b = a;
    b.out[0] = (uint16_t*)a.out[half] + e * step_out;
    finish4<T, OUT_PLAIN, 0>(b, 0, row - half * (int64_t)a.part_rows, c, v);
  }
}

// Few rows: the form of dense_rows.h, a block for 16 outputs and 16 rows of one
// expert.  Bound by reading the weights: 32 rows of 16 experts, 2048 -> 4096 gated,
// 49 us where the caches hold part of them, 99 from memory (5.1 TB/s).
template <class T, int H, int NW>
__global__ __launch_bounds__(NW * 64) void moe_rows_kernel(RowsArgs a, Groups g, int64_t step_w) {
  __shared__ v4u xs[16 * rows_ld(NW) / 8];
  const GroupPieces pieces(g, 16);
  // as in dense_rows_kernel, the pieces in place of the token tiles
  const uint32_t many = pieces.total, nt = many ? blockIdx.x / (8ull * many) * 8 + blockIdx.x % 8 : a.tiles_n;
  if (nt >= (uint32_t)a.tiles_n) return;
  int e, piece;
  pieces.find(g, blockIdx.x / 8 % many, e, piece);
  const GroupRows rows = group_rows(g, e);
  const int64_t first = __builtin_amdgcn_readfirstlane(rows.first);
  a.m = __builtin_amdgcn_readfirstlane(rows.count);
  a.x += first * a.ld_x;
  a.y += first * a.ld_y;
  if (a.pre) a.pre += first * 2 * a.ld_pre;
#pragma unroll
  for (int h = 0; h < H; ++h) a.w[h] = (const uint16_t*)a.w[h] + e * step_w;
  dense_rows_tile<T, Dense16, H, 1, NW>(a, xs, nt, piece);
}

int64_t few_blocks(int rows, int groups, int outputs) {
  return round_up(ceil_div(outputs, 16), 8) * GroupPieces::most(rows, groups, 16);
}
template <class T, int H>
int run_few(RowsArgs& a, const Groups& g, int64_t step_w, hipStream_t s) {
  constexpr int NW = 8;
  a.tiles_n = ceil_div(a.n, 16);
  moe_rows_kernel<T, H, NW><<<(unsigned)few_blocks(g.rows, g.n, a.n), NW * 64, 0, s>>>(a, g, step_w);
  return hip_status();
}

template <class T, class SR, class SC, int OUT, int B>
int run_tiles(GemmArgs& a, const Groups& g, int64_t step_c, hipStream_t s) {
  a.tiles_c = ceil_div(a.cols, OUT == OUT_GATED ? B / 2 : B);
  int64_t blocks = GroupPieces::most(g.rows, g.n, B) * a.tiles_c * a.parts;
  if (B == 256) blocks += 256;  // parts of the last tiles
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;  // 2^31 threads
  a.rows = a.part_rows = g.rows;
  a.ld_part = (int)round_up(a.cols, 4);
  if (B != 256 && a.parts == 1) a.part = nullptr;
  moe_gemm_kernel<T, SR, SC, OUT, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a, g, step_c);
  if (B == 256) {
    moe_tail_kernel<T, OUT><<<128 * 16, 256, 0, s>>>(a, g);  // more tiles than 128 are not split
  } else if (a.parts > 1) {
    const int64_t n = (int64_t)g.rows * (a.ld_part / 4);
    moe_join_kernel<T, OUT><<<(unsigned)(n < (1 << 20) ? (n + 255) / 256 : 4096), 256, 0, s>>>(a, g);
  }
  return hip_status();
}
template <class T, class SR, class SC, int B>
int run_tiles_w(GemmArgs& a, const Groups& g, int size, int64_t step_out, hipStream_t s) {
  // with a tile for each compute unit, an expert twice as long as a piece is not worth cutting
  const int uncut = size < 0x3fffff00 && (int64_t)ceil_div(a.rows, 256) * ceil_div(a.cols, 256) * a.halves * g.n >= 256 ? 2 * size : size;
  a.tiles_r = ceil_div(a.rows, B);
  a.tiles_c = ceil_div(a.cols, B);
  const int64_t blocks = ((int64_t)g.rows / size + g.n) * a.tiles_r * a.halves * a.tiles_c;
  if (blocks >= (1 << 22)) return QCONV_EUNSUPPORTED;
  a.part_rows = a.rows;
  a.ld_part = (int)round_up(a.cols, 4);
  moe_gemm_w_kernel<T, SR, SC, B><<<(unsigned)blocks, B / 64 * 128, 0, s>>>(a, g, size, uncut, step_out);
  if (g.rows > size) {
    const int64_t n = (int64_t)a.halves * a.rows * (a.ld_part / 4);
    const int several = g.rows / size < g.n ? g.rows / size : g.n;
    moe_join_w_kernel<T><<<dim3((unsigned)(n < (1 << 17) ? (n + 255) / 256 : 512), several), 256, 0, s>>>(a, g, size, uncut, step_out);
  }
  return hip_status();
}

// Rows of the batch by the weights' rows (CCOL false) or columns.
template <class T, bool CCOL, int OUT>
int run_rows_t(GemmArgs& a, const Groups& g, int64_t step_c, const GemmPlan& p, bool aligned, hipStream_t s) {
  a.parts = p.parts;
  constexpr bool PAIR = OUT == OUT_GATED;
  constexpr int KS = CCOL ? 32 : 64;
  if (!aligned)
    return run_tiles<T, Stage16<KS, 128, 256, 0, false, false, false>, Stage16<KS, 128, 256, 1, CCOL, false, PAIR>, OUT,
                     128>(a, g, step_c, s);
  if (p.tile == 256)
    return run_tiles<T, Stage16<KS, 256, 512, 0, false, true, false>, Stage16<KS, 256, 512, 1, CCOL, true, PAIR>, OUT,
                     256>(a, g, step_c, s);
  return run_tiles<T, Stage16<KS, 128, 256, 0, false, true, false>, Stage16<KS, 128, 256, 1, CCOL, true, PAIR>, OUT,
                   128>(a, g, step_c, s);
}
template <bool CCOL, int OUT>
int run_rows(int dtype, GemmArgs& a, const Groups& g, int64_t step_c, const GemmPlan& p, bool aligned, hipStream_t s) {
  return dtype == QCONV_F16 ? run_rows_t<F16, CCOL, OUT>(a, g, step_c, p, aligned, s)
                            : run_rows_t<BF16, CCOL, OUT>(a, g, step_c, p, aligned, s);
}
template <class T>
int run_weights_t(GemmArgs& a, const Groups& g, int64_t step_out, int tile, int size, bool aligned, hipStream_t s) {
  if (!aligned)
    return run_tiles_w<T, Stage16<32, 128, 256, 0, true, false, false>, Stage16<32, 128, 256, 1, true, false, false>,
                       128>(a, g, size, step_out, s);
  if (tile == 256)
    return run_tiles_w<T, Stage16<32, 256, 512, 0, true, true, false>, Stage16<32, 256, 512, 1, true, true, false>,
                       256>(a, g, size, step_out, s);
  return run_tiles_w<T, Stage16<32, 128, 256, 0, true, true, false>, Stage16<32, 128, 256, 1, true, true, false>, 128>(
      a, g, size, step_out, s);
}

// The products whose rows are the batch's: tiles of 256 x 256 where there are
// enough for the 256 compute units and the experts' rows, on average, fill three
// quarters of one, or fewer with long sums, which all count as last ones then (gx of
// 4096 rows of 8 experts, 4096 -> 1024, with its slopes: 142 us against 208 in small
// tiles), else 128 x 128.  Few of those are split as in gemm_plan, and until
// there are two for each unit as long as each part keeps 1024 products: us of the linear
// forward with a block and with two for each unit, weights from memory: 700 rows of 8
// experts 4096 -> 1024 42.3 and 31.7, 600 of 3 4096 -> 4096 66.6 and 51.7; with fewer
// products each, 941 of 2 1024 -> 2456 17.4 and 21.9.
GemmPlan plan_rows(const qconv_moe_desc& d, int cols, int64_t products, bool gated, bool aligned) {
  auto tiles = [&](int b) {
    const int64_t n = GroupPieces::most(d.rows, d.groups, b) * ceil_div(cols, gated ? b / 2 : b);
    return n > 0 ? n : 1;
  };
  // the tiles there will be if half of the experts' last ones are full
  const int64_t likely = (d.rows / 256 * 2 + (int64_t)d.groups) * ceil_div(cols, gated ? 128 : 256) / 2;
  const bool long_sums = likely > 0 && likely <= 256 && 256 / likely * likely >= 192 && products / (256 / likely) >= 2048;
  if (aligned && d.rows >= 192 * (int64_t)d.groups && (tiles(256) >= 256 || long_sums))
    return {256, 1, (size_t)256 * TAIL_TILE * 4};
  const int64_t small = tiles(128);
  int64_t parts = small >= 192 ? 1 : 256 / small;
  if (parts > products / 512) parts = products / 512;
  const int64_t two = 512 / small < products / 1024 ? 512 / small : products / 1024;
  parts = parts > two ? parts : two;
  if (parts <= 1) return {128, 1, 0};
  return {128, (int)parts, (size_t)parts * (gated ? 2 : 1) * d.rows * round_up(cols, 4) * 4};
}

// Weight gradients: the tile, and the rows of a piece.  Enough tiles: an expert's rows
// are one piece.  Otherwise pieces make about twice as many tiles as fit the chip, or
// more where experts are uneven, and are long enough to be worth their sums' way
// through memory (8192 rows of 8 experts, 2048 -> 2048: 105 us whole, 121 in pieces of
// 1536 rows; 32768 rows of 16, of unequal shares, 1024 -> 1024: 304 us
// whole, 121 in pieces of 1536).
struct PlanW {
  int tile, size;
  size_t bytes;
};
PlanW plan_weights(const qconv_moe_desc& d, bool gated, bool aligned) {
  const int halves = gated ? 2 : 1;
  auto tiles = [&](int b) { return (int64_t)ceil_div(d.f, b) * ceil_div(d.k, b) * halves; };
  const int tile = aligned && tiles(256) * d.groups >= 256 ? 256 : 128;
  const int64_t per = tiles(tile), slots = tile == 256 ? 256 : 512;
  if (per * d.groups >= 4 * slots) return {tile, 0x7fffff00, 0};
  int64_t size = round_up(d.rows * per / (2 * slots), 64);
  const int least = tile == 256 ? 1536 : 512;
  size = size < least ? least : size < 0x7fffff00 ? size : 0x7fffff00;
  // a tile for each unit, and even all rows in one expert would be short
  if (per * d.groups >= slots && d.rows <= 3 * size) return {tile, 0x7fffff00, 0};
  return {tile, (int)size, d.rows > size ? (size_t)(2 * ((d.rows + size - 1) / size) * halves * d.f * round_up(d.k, 4) * 4) : 0};
}

// The rows that go forward without tiles.  Tiles read the same weights through LDS
// and are slower at it while there is less than a tile of rows for each expert; the
// blocks without tiles read x for every 16 outputs.  us here and there, gated, weights
// from memory (both with 10 us of a call's own):
//   16 experts 2048 -> 4096   99 and 128 at 32 rows, 109 and 132 at 128, 136 and 132 at 256
//   64 experts 2048 -> 1024   73 and 101 at 64, 106 and 131 at 256, 141 and 134 at 1024
//   64 experts 512 -> 512     12.4 and 15.5 at 32, 17.4 and 16.6 at 64, 24 and 19 at 256
// Tiles take more outputs, too, than blocks of 16 outputs may be launched for (2^31 threads).
bool few_rows(const qconv_moe_desc& d) {
  if (few_blocks(d.rows, d.groups, d.f) >= (1 << 22)) return false;
  const int many = d.k < 1024 ? 32 : 4 * d.groups;
  return d.rows <= (d.k >= 1024 && many < 64 ? 64 : many);
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

size_t moe_forward_bytes(const qconv_moe_desc& d, bool gated) {
  if (few_rows(d)) return 0;
  const size_t p = plan_rows(d, d.f, d.k, gated, false).bytes, q = plan_rows(d, d.f, d.k, gated, true).bytes;
  return copies_bytes(d, gated, true) + (p > q ? p : q);
}

int launch_moe_forward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                       void* h, float* pre, void* ws, hipStream_t s) {
  if (d.rows == 0) return QCONV_OK;
  const Groups g = {offsets, d.groups, d.rows};
  if (few_rows(d)) {
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
    r.n = d.f;
    r.k = d.k;
    r.act = d.act;
    const int64_t step = (int64_t)d.f * d.ld_w;
    if (wu) return d.dtype == QCONV_F16 ? run_few<F16, 2>(r, g, step, s) : run_few<BF16, 2>(r, g, step, s);
    return d.dtype == QCONV_F16 ? run_few<F16, 1>(r, g, step, s) : run_few<BF16, 1>(r, g, step, s);
  }
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
  const GemmPlan p = plan_rows(d, d.f, d.k, wu, aligned);
  a.part = (float*)((char*)ws + copies_bytes(d, wu, true));
  return wu ? run_rows<false, OUT_GATED>(d.dtype, a, g, step, p, aligned, s)
            : run_rows<false, OUT_PLAIN>(d.dtype, a, g, step, p, aligned, s);
}

size_t moe_backward_bytes(const qconv_moe_desc& d, bool gated) {
  size_t most = 0;
  for (bool aligned : {false, true}) {
    const size_t p = plan_rows(d, d.k, (gated ? 2 : 1) * (int64_t)d.f, false, aligned).bytes;
    const size_t q = plan_weights(d, gated, aligned).bytes;
    most = p > most ? p : most;
    most = q > most ? q : most;
  }
  return copies_bytes(d, gated, false) + factor_bytes(d, gated) + most;
}

int launch_moe_backward(const qconv_moe_desc& d, const void* x, const void* wg, const void* wu, const int* offsets,
                        const float* pre, const void* gh, void* gx, void* gwg, void* gwu, void* ws, hipStream_t s) {
  const Groups g = {offsets, d.groups, d.rows};
  const int fp = (int)round_up(d.f, 8);
  Operand ox = {(const uint16_t*)x, d.ld_x}, og = {(const uint16_t*)wg, d.ld_w};
  Operand ou = wu ? Operand{(const uint16_t*)wu, d.ld_w} : og;
  uint16_t* factors = (uint16_t*)((char*)ws + copies_bytes(d, wu, false));
  float* part = (float*)((char*)factors + factor_bytes(d, wu));
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
    a.part = part;
    const GemmPlan p = plan_rows(d, d.k, a.segments * (int64_t)d.f, false, aligned);
    rc = run_rows<true, OUT_PLAIN>(d.dtype, a, g, (int64_t)d.f * og.ld, p, aligned, s);
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
    a.part = part;
    const PlanW p = plan_weights(d, wu, aligned);
    const int64_t step = (int64_t)d.f * d.k;
    rc = d.dtype == QCONV_F16 ? run_weights_t<F16>(a, g, step, p.tile, p.size, aligned, s)
                              : run_weights_t<BF16>(a, g, step, p.tile, p.size, aligned, s);
  }
  return rc;
}

}  // namespace qc
