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

// A tile's expert and first slot; end: the expert's.
struct RowTile { int e, s0, end; };

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
__device__ __forceinline__ Slots expert_slots(const ExpertTiles &x, int e) {
  const int b = min(max(x.offsets[e], 0), x.P), c = min(max(x.offsets[e + 1], b), x.P);
  return {b, c - b > x.above && c - b <= x.most ? c : b};
}

// The experts' row tiles of kRows slots counted by a wave, each lane having the same number
// of consecutive experts.
template <int kRows>
struct TileCount {
  int per, mine, incl, total;
  __device__ __forceinline__ explicit TileCount(const ExpertTiles &x) {
    const int lane = threadIdx.x & 63;
    per = (x.E + 63) / 64;
    mine = 0;
    for (int i = 0; i < per; ++i) {
      const int e = lane * per + i;
      if (e < x.E) {
        const Slots s = expert_slots(x, e);
        mine += (s.end - s.begin + kRows - 1) / kRows;
      }
    }
    incl = wave_inclusive_sum(mine);
    total = __builtin_amdgcn_readlane(incl, 63);
  }
  // The expert of row tile t (below total), its slots and its first row tile; -1 if none.
  __device__ __forceinline__ int find(const ExpertTiles &x, int t, Slots &s, int &first) const {
    const int l = __builtin_ctzll(__ballot(incl > t));
    first = __builtin_amdgcn_readlane(incl - mine, l);
    for (int e = l * per, last = min(e + per, x.E); e < last; ++e) {
      s = expert_slots(x, e);
      const int tiles = (s.end - s.begin + kRows - 1) / kRows;
      if (t < first + tiles) return e;
      first += tiles;
    }
    return -1;
  }
};

// Tile blockIdx.x of the experts' tiles of kRows slots by ntn column tiles; false past the
// last.  The tiles of one XCD (workgroups are dealt to the 8 XCDs round robin) are
// consecutive, an expert's walked in groups of GM row tiles, so that the tiles that run
// together share rows and weights in that XCD's L2.
template <int kRows, int GM>
__device__ __forceinline__ bool expert_tile(const ExpertTiles &x, int ntn, RowTile &tile, int &tn) {
  const TileCount<kRows> count(x);
  const int tiles = count.total * ntn, chunk = (tiles + 7) / 8;
  const int t = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= chunk || t >= tiles) return false;
  Slots s;
  int first;
  if ((tile.e = count.find(x, t / ntn, s, first)) < 0) return false;
  const int at = t - first * ntn, ntm = (s.end - s.begin + kRows - 1) / kRows;
  const int group = at / (GM * ntn), size = min(ntm - group * GM, GM);
  const int in = at - group * GM * ntn;
  tile.s0 = s.begin + (group * GM + in % size) * kRows;
  tile.end = s.end;
  tn = in / size;
  return true;
}

// The activation row of a slot, as an unsigned number: an index outside the activations is
// at least their number.
__device__ __forceinline__ uint32_t expert_row(const ExpertTiles &x, int64_t slot) {
  return x.rows ? (uint32_t)x.rows[slot] : (uint32_t)slot;
}

}  // namespace
}  // namespace rfq
