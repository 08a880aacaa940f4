// Row tiles of slots that are sorted by expert, from the offsets on the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rfq {

// The slots of the experts a launch multiplies: those with more than `above` and at most
// `most` slots (the others are another launch's).
struct ExpertTiles {
  const int32_t *offsets;   // [E + 1], not decreasing; cut to [0, P]
  const int32_t *rows;      // [P] activation row of a slot, or nullptr: its own number
  int E, P, above, most;
};

// A tile's expert, first slot and column tile; end: the expert's.
struct RowTile { int e, s0, end, tn; };

namespace {

// Inclusive prefix sum over the wave's lanes: steps of 1, 2, 4 and 8 lanes inside rows of
// 16, then the rows' sums passed on.
__device__ __forceinline__ int wave_inclusive_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

struct Slots { int begin, end; };
// The slots between two offsets, none where they are another launch's.
__device__ __forceinline__ Slots slots_between(const ExpertTiles &x, int from, int to) {
  const int b = min(max(from, 0), x.P), c = min(max(to, b), x.P);
  return {b, c - b > x.above && c - b <= x.most ? c : b};
}

// The experts' row tiles of kRows slots counted by a wave, each lane having the same number
// of consecutive experts: up to kHeld of them (256 experts) with their offsets in registers,
// which a workgroup then finds its tile in after one round trip to memory.
template <int kRows>
struct TileCount {
  static constexpr int kHeld = 4;
  int per, mine, incl, total, held[kHeld + 1];
  static __device__ __forceinline__ int tiles(const Slots &s) {
    return (s.end - s.begin + kRows - 1) / kRows;
  }
  __device__ __forceinline__ explicit TileCount(const ExpertTiles &x) {
    const int lane = threadIdx.x & 63;
    per = (x.E + 63) / 64;
    const int e0 = min(lane * per, x.E);
    mine = 0;
#pragma unroll
    for (int i = 0; i <= kHeld; ++i) held[i] = x.offsets[min(e0 + min(i, per), x.E)];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) mine += tiles(slots_between(x, held[i], held[i + 1]));
    if (per > kHeld) {
      mine = 0;
      for (int i = 0; i < per; ++i) {
        const int e = min(e0 + i, x.E);
        mine += tiles(slots_between(x, x.offsets[e], x.offsets[min(e + 1, x.E)]));
      }
    }
    incl = wave_inclusive_sum(mine);
    total = __builtin_amdgcn_readlane(incl, 63);
  }
  // The expert of row tile t (below total), its slots and its first row tile; -1 if none.
  __device__ __forceinline__ int find(const ExpertTiles &x, int t, Slots &s, int &first) const {
    const uint64_t past = __ballot(incl > t);
    if (!past) return -1;
    const int l = __builtin_ctzll(past);
    first = __builtin_amdgcn_readlane(incl - mine, l);
    int e = l * per;
    if (per <= kHeld) {
      int from = __builtin_amdgcn_readlane(held[0], l);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int to = __builtin_amdgcn_readlane(held[i + 1], l);
        s = slots_between(x, from, to);
        const int n = tiles(s);
        if (t < first + n) return e + i;
        first += n;
        from = to;
      }
      return -1;
    }
    for (const int last = min(e + per, x.E); e < last; ++e) {
      s = slots_between(x, x.offsets[e], x.offsets[e + 1]);
      const int n = tiles(s);
      if (t < first + n) return e;
      first += n;
    }
    return -1;
  }
};

// Tile `bid` (a workgroup's number) of the experts' tiles of kRows slots by ntn column tiles;
// false past the last.  An expert's tiles are walked in groups of GM row tiles, so that those
// that run together share rows and weights.  SPREAD: workgroups are dealt to the 8 XCDs round
// robin, and each XCD gets consecutive tiles, which share them in its L2 (half of 128 experts'
// products for 8192 tokens, 256 x 256 tiles: 150 us without, 139 with it).
template <int kRows, int GM, bool SPREAD>
__device__ __forceinline__ bool expert_tile(const ExpertTiles &x, int bid, int ntn, RowTile &tile) {
  const TileCount<kRows> count(x);
  const int tiles = count.total * ntn, chunk = (tiles + 7) / 8;
  const int t = SPREAD ? (bid & 7) * chunk + (bid >> 3) : bid;
  if ((SPREAD && (bid >> 3) >= chunk) || t >= tiles) return false;
  Slots s;
  int first;
  if ((tile.e = count.find(x, t / ntn, s, first)) < 0) return false;
  const int at = t - first * ntn, ntm = TileCount<kRows>::tiles(s);
  const int group = at / (GM * ntn), size = max(min(ntm - group * GM, GM), 1);
  const int in = at - group * GM * ntn;
  tile.s0 = s.begin + (group * GM + in % size) * kRows;
  tile.end = s.end;
  tile.tn = in / size;
  // (With decreasing offsets the counts can pass 32 bits: nothing is read or written outside
  // then either.)
  return tile.s0 >= s.begin && tile.s0 < s.end && tile.tn >= 0 && tile.tn < ntn;
}

// The activation row of a slot, as an unsigned number: an index outside the activations is
// at least their number.
__device__ __forceinline__ uint32_t expert_row(const ExpertTiles &x, int64_t slot) {
  return x.rows ? (uint32_t)x.rows[slot] : (uint32_t)slot;
}

}  // namespace
}  // namespace rfq
