// moe_groups.h -- which rows of a batch belong to which weight: offsets[g] ..
// offsets[g + 1] are the rows of group g, known to the device alone.
#pragma once

#include "dense.h"

namespace qc {

struct Groups {
  const int* offsets;  // [n + 1]
  int n;
  int rows;  // rows there are: whatever offsets says, none past them are touched
};

struct GroupRows {
  int first, count;
};
__device__ __forceinline__ GroupRows group_rows(const Groups& g, int e) {
  const int lo = g.offsets[e], hi = g.offsets[e + 1];
  const int first = lo < 0 ? 0 : lo < g.rows ? lo : g.rows, last = hi < g.rows ? hi : g.rows;
  return {first, last > first ? last - first : 0};
}

// Inclusive sums over the wave's lanes.
__device__ __forceinline__ int wave_sums(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// The pieces of `size` rows that the groups' rows fall into, numbered group
// after group: the host, which does not know the offsets, launches most() of them
// and a block looks its piece up by itself: each wave, a lane its share of the groups,
// one after the other.  That is about 1 us up to 256 groups and bounds the kernels past
// some hundred: us at 16, 256, 1024 and 4096 groups, 64 tokens with adapters of rank 8,
// 1024 -> 1024, 6.7, 7.0, 8.7 and 19.8; 4096 rows 128 -> 128 forward 8.1, 7.8, 19 and
// 152, their weight gradients 11.4, 12.0, 57 and 485.  With `empty` a group without
// rows has a piece, too; with `several` only groups of more than one piece count, as one.
struct GroupPieces {
  static int64_t most(int rows, int groups, int size) { return rows / size + (groups < rows ? groups : rows); }

  int size, per;  // groups per lane
  bool empty, several;
  int upto;       // pieces of the groups up to and with this lane's
  int total;

  // At most MOST, far above what is ever launched: sums over offsets of no order, where
  // groups share rows, stay inside an int.
  static constexpr int MOST = 1 << 24;
  __device__ __forceinline__ int of(const Groups& g, int e) const {
    if (e >= g.n) return 0;
    const int rows = group_rows(g, e).count;
    if (several) return rows > size ? 1 : 0;
    const int n = rows > 0 ? (rows - 1) / size + 1 : empty ? 1 : 0;
    return n < MOST ? n : MOST;
  }
  __device__ __forceinline__ GroupPieces(const Groups& g, int size_, bool empty_ = false, bool several_ = false)
      : size(size_), empty(empty_), several(several_) {
    const int lane = threadIdx.x & 63;
    per = (g.n + 63) / 64;
    int mine = 0;
    for (int i = 0; i < per; ++i) mine += of(g, lane * per + i);
    upto = wave_sums(mine < MOST ? mine : MOST);
    total = __builtin_amdgcn_readlane(upto, 63);
  }
  // The group of piece p < total, and the piece's number in it.
  __device__ __forceinline__ void find(const Groups& g, int p, int& group, int& piece) const {
    const int lane = threadIdx.x & 63;
    int l = __popcll(__ballot(upto <= p));
    int before = l ? __builtin_amdgcn_readlane(upto, l - 1) : 0;
    group = l;
    if (per > 1) {  // at most 64 groups of that lane's, one in each
      const int e = l * per + lane, sums = wave_sums(lane < per ? of(g, e) : 0);
      const int in = __popcll(__ballot(before + sums <= p));
      before += in ? __builtin_amdgcn_readlane(sums, in - 1) : 0;
      group = l * per + in;
    }
    group = __builtin_amdgcn_readfirstlane(group);
    piece = __builtin_amdgcn_readfirstlane(p - before);
  }
};

// The rows of a piece where groups of up to `most` rows need not be cut: `size`, or
// all of them.
__device__ __forceinline__ int group_size(const Groups& g, int size, int most) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int e = lane; e < g.n; e += 64) {
    const int c = group_rows(g, e).count;
    n = c > n ? c : n;
  }
  return __ballot(n > most) ? size : 0x7fffff00;
}

// The p-th largest of at most 64 groups (equal ones in their order).
__device__ __forceinline__ int group_by_size(const Groups& g, int p) {
  const int lane = threadIdx.x & 63, mine = lane < g.n ? group_rows(g, lane).count : -1;
  int before = 0;
  for (int e = 0; e < g.n; ++e) {
    const int other = __builtin_amdgcn_readlane(mine, e);
    before += other > mine || (other == mine && e < lane) ? 1 : 0;
  }
  return __builtin_ctzll(__ballot(lane < g.n && before == p));
}

// Where the sums over piece `piece` of a group of several are kept, if the group's
// rows start at `first`: pieces of one group start `size` rows apart, so at most two
// of groups with several start in the same `size` rows, and of these one is its
// group's first.  2 * ceil(rows / size) places do.
__device__ __forceinline__ int64_t group_part(int64_t first, int piece, int size) {
  return 2 * (first / size + piece) + (piece == 0 ? 1 : 0);
}

}  // namespace qc
