// Pairs (token, choice) sorted by expert, and the way back: with e_p the expert of pair p
// (its number less `first`; outside [0, E) the pair is dropped),
//     slot of p = offsets[e_p] + (pairs before p with the same expert),
//     rows[slot] = p / k,  offsets[e] = pairs with an expert below e.
//
// A counting sort, stable and without an order left to chance: a workgroup of 16 waves
// counts its pairs per expert and wave, turns the counts into first slots by prefix sums
// over experts and waves, and places the pairs of 64 lanes at a time: a lane's rank is the
// number of lower lanes whose expert has the same bits (one ballot per bit).  The counters
// are LDS integers, whose sums do not depend on the order of the additions.
//
// Up to kOneGroup pairs one workgroup does all of it.  Beyond, workgroups count their
// pairs in one launch (workspace [groups][E]), and in a second one each repeats the prefix sums
// over all groups before it places its own pairs: no workgroup waits for another.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "experts.h"
#include "experts_device.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int64_t kOneGroup = 8192;           // pairs
constexpr int64_t kMaxGroups = 64;
constexpr int kHeld = 4;
constexpr int kBatch = 16;                    // groups whose counts are loaded together

int64_t pairs_per_group(int64_t P) {
  const int64_t even = (P + kMaxGroups - 1) / kMaxGroups;
  return std::max<int64_t>(2048, (even + kThreads - 1) / kThreads * kThreads);
}

struct Pairs {
  const int32_t *experts;
  int64_t P, first;
  int E;
  // The pair's expert here, E where it is dropped or past the last.
  __device__ __forceinline__ int at(int64_t p) const {
    if (p >= P) return E;
    const int64_t e = (int64_t)experts[p] - first;
    return e >= 0 && e < E ? (int)e : E;
  }
};

// The pairs [p0, p1) that this wave places; p0 a multiple of 64 from the group's start.
struct Range { int64_t p0, p1; };
__device__ __forceinline__ Range wave_range(int64_t g0, int64_t g1) {
  const int wave = threadIdx.x >> 6;
  const int64_t per = ((g1 - g0 + 63) / 64 + kWaves - 1) / kWaves * 64;
  const int64_t p0 = min(g0 + wave * per, g1);
  return {p0, min(p0 + per, g1)};
}

__global__ __launch_bounds__(kThreads) void expert_count_kernel(Pairs pairs, int64_t per_group,
                                                                int32_t *__restrict__ counts) {
  __shared__ int count[kMaxExperts];
  const int E = pairs.E;
  for (int e = threadIdx.x; e < E; e += kThreads) count[e] = 0;
  __syncthreads();
  const int64_t g0 = (int64_t)blockIdx.x * per_group, g1 = min(g0 + per_group, pairs.P);
  for (int64_t p = g0 + threadIdx.x; p < g1; p += kThreads) {
    const int e = pairs.at(p);
    if (e < E) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) counts[(int64_t)blockIdx.x * E + e] = count[e];
}

// counts == nullptr: one workgroup, all pairs.  Dynamic LDS: kWaves * E counters.
__global__ __launch_bounds__(kThreads) void expert_place_kernel(
    Pairs pairs, int k, int64_t per_group, const int32_t *__restrict__ counts,
    int32_t *__restrict__ offsets, int32_t *__restrict__ rows, int32_t *__restrict__ slots) {
  extern __shared__ int next[];                    // [kWaves][E]: the wave's next slots
  __shared__ int part[kWaves];
  __shared__ int sums[2][kThreads];
  const int E = pairs.E, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t g0 = (int64_t)blockIdx.x * per_group, g1 = min(g0 + per_group, pairs.P);
  const Range mine = wave_range(g0, g1);

  for (int i = tid; i < kWaves * E; i += kThreads) next[i] = 0;
  __syncthreads();
  // The wave's first kHeld chunks of 64 pairs stay in registers.
  int held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int64_t p = mine.p0 + 64 * i + lane;
    held[i] = p < mine.p1 ? pairs.at(p) : E;
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (held[i] < E) atomicAdd(&next[wave * E + held[i]], 1);
  for (int64_t p = mine.p0 + 64 * kHeld + lane; p < mine.p1; p += 64) {
    const int e = pairs.at(p);
    if (e < E) atomicAdd(&next[wave * E + e], 1);
  }
  __syncthreads();

  // Expert e = tid: its pairs in all groups and in those before this one.  (A thread adds
  // those of part of the groups: with all of them in one chain of loads 32768 tokens of 8
  // choices among 256 experts took 33 us.)
  int all = 0, before = 0;
  if (counts) {
    const int groups = gridDim.x, me = blockIdx.x, ways = kThreads / E;
    const int e = tid % E, way = tid / E;
    const int end = way < ways ? groups * (way + 1) / ways : 0;
    for (int g = way < ways ? groups * way / ways : 0; g < end; g += kBatch) {
      int c[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) c[b] = counts[(int64_t)min(g + b, end - 1) * E + e];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        all += g + b < end ? c[b] : 0;
        before += g + b < min(end, me) ? c[b] : 0;
      }
    }
    sums[0][tid] = all;
    sums[1][tid] = before;
    __syncthreads();
    all = before = 0;
    for (int w = 0; tid < E && w < ways; ++w) {
      all += sums[0][w * E + tid];
      before += sums[1][w * E + tid];
    }
  } else if (tid < E) {
    for (int w = 0; w < kWaves; ++w) all += next[w * E + tid];
  }
  const int incl = wave_inclusive_sum(all);
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int base = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    base += w < wave ? part[w] : 0;
    total += part[w];
  }
  if (tid < E) {
    const int first = base + incl - all;
    if (blockIdx.x == 0) offsets[tid] = first;
    int at = first + before;
    int c[kWaves];           // (Read before the first is written: one round trip.)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) c[w] = next[w * E + tid];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      next[w * E + tid] = at;
      at += c[w];
    }
  }
  if (tid == 0 && blockIdx.x == 0) offsets[E] = total;
  __syncthreads();

  const int bits = 32 - __builtin_clz(E);          // E itself stands for a dropped pair
  auto place = [&](int64_t p, int e) {
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const bool bit = (e >> b) & 1;
      const uint64_t m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    int slot = -1;
    if (e < E) {
      // One wave's LDS accesses are served in order: all lanes read before the last of
      // an expert writes.
      const int at = next[wave * E + e];
      slot = at + rank;
      if ((same >> lane) == 1) next[wave * E + e] = slot + 1;
      rows[slot] = (int)((uint32_t)p / (uint32_t)k);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (p < mine.p1) slots[p] = slot;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (mine.p0 + 64 * i < mine.p1) place(mine.p0 + 64 * i + lane, held[i]);
  for (int64_t c = mine.p0 + 64 * kHeld; c < mine.p1; c += 64)
    place(c + lane, c + lane < mine.p1 ? pairs.at(c + lane) : E);
  // Slots that no pair has.
  for (int64_t p = max((int64_t)total, g0) + tid; p < g1; p += kThreads) rows[p] = -1;
}

}  // namespace

int64_t expert_sort_workspace(int64_t T, int64_t k, int64_t E) {
  const int64_t P = T * k;
  if (P <= kOneGroup) return 0;
  const int64_t per = pairs_per_group(P);
  return (P + per - 1) / per * E * 4;
}

hipError_t launch_expert_sort(const int32_t *experts, int64_t T, int k, int64_t first, int E,
                              int32_t *offsets, int32_t *rows, int32_t *slots, void *workspace,
                              int64_t workspace_bytes, hipStream_t stream) {
  const int64_t P = T * k, need = expert_sort_workspace(T, k, E);
  const Pairs pairs{experts, P, first, E};
  const unsigned lds = (unsigned)(kWaves * E * 4);
  static std::atomic<bool> limit_done[kMaxDevices];
  hipError_t e = set_lds_limit(limit_done, reinterpret_cast<const void *>(expert_place_kernel),
                               (int)(kWaves * kMaxExperts * 4));
  if (e != hipSuccess) return e;
  if (need == 0 || workspace_bytes < need) {
    expert_place_kernel<<<1, kThreads, lds, stream>>>(pairs, k, P, nullptr, offsets, rows, slots);
    return hipGetLastError();
  }
  const int64_t per = pairs_per_group(P);
  const unsigned groups = (unsigned)((P + per - 1) / per);
  int32_t *counts = static_cast<int32_t *>(workspace);
  expert_count_kernel<<<groups, kThreads, 0, stream>>>(pairs, per, counts);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  expert_place_kernel<<<groups, kThreads, lds, stream>>>(pairs, k, per, counts, offsets, rows, slots);
  return hipGetLastError();
}

}  // namespace rfq
