// Block tables and slot maps of a paged key/value cache, from the requests'
// lengths on the device.
//
// With held = ceil(ctx / page), need = ceil((ctx + new) / page) and the exclusive
// prefix sums F of need - held and S of new over the requests, the n-th new token
// of request b (row S_b + n) stands at p = ctx_b + n, in block p / page of the
// request; the block is the table's where p / page < held_b, else the one taken as
// number F_b + p / page - held_b.  Every taken block holds exactly one new token at
// its start, so the token with p % page == 0 writes the table entry and nothing
// is searched twice (but for tokens that the call's `tokens` leaves out).
//
// The work is two int32 in and a few out per request and two out per token: a few
// hundred KB at most, so a call costs its launch and its chain of dependent
// loads.  Every workgroup therefore repeats the prefix sums of all requests
// (a few values a thread, 16 bytes a request from L2) instead of a second launch
// that would wait for a first; no workgroup reads what another writes.  Measured: one new
// token of each of 16 requests 3.5 us, 2000 requests with 128540 new tokens 7.7 us; the blocks
// of 500 requests given back in 4.4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "kv.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

// Workgroups of 256 work items, or with many requests of 1024: a request's lengths are a
// round trip to L2 apart where a thread has several (2000 requests, 128540 tokens: 12.7 us
// with 256, 7.7 with 1024 and loads in fours).
constexpr int kFewThreads = 256, kManyThreads = 1024;
constexpr int kTokensPerGroup = 1024;
constexpr int kBatch = 4;                   // requests whose lengths are loaded together

__device__ __forceinline__ int64_t wave_inclusive(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// Exclusive prefix over the workgroup's threads; total: the sum.  part: a value of LDS
// for each wave, that nothing else uses until the next barrier.
template <int kThreads>
__device__ __forceinline__ int64_t group_exclusive(int64_t v, int64_t *part, int64_t &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t incl = wave_inclusive(v);
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  return before + incl - v;
}

__device__ __forceinline__ int32_t saturated(int64_t v) {
  return v > INT32_MAX ? INT32_MAX : (int32_t)v;
}
__device__ __forceinline__ int64_t clamped(int64_t v, int64_t lo, int64_t hi) {
  return v < lo ? lo : (v > hi ? hi : v);
}

// The last index b in [0, n) with start[b] <= t (start[0] == 0, not decreasing).
__device__ __forceinline__ int owner(const int32_t *start, int n, int64_t t) {
  int lo = 0, hi = n;                       // start[lo] <= t, start[hi] > t or hi == n
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void block_assign_kernel(
    const int32_t *__restrict__ ctx_lens, const int32_t *__restrict__ new_lens, int B,
    int32_t *tables, int64_t width, const int32_t *__restrict__ free_blocks, int64_t n_free,
    const int32_t *__restrict__ free_count, int page_shift, int64_t tokens,
    int32_t *__restrict__ slots, int32_t *__restrict__ positions, int32_t *__restrict__ seq_lens,
    int32_t *__restrict__ query_starts, int32_t *__restrict__ counts) {
  extern __shared__ int32_t lds[];
  int32_t *start = lds;                     // [B] first token of each request
  int32_t *first = lds + B;                 // [B] blocks taken before it; -1: refused
  __shared__ int64_t part[3][kThreads / 64];
  const int tid = threadIdx.x, per = (B + kThreads - 1) / kThreads;
  const int b0 = tid * per, b1 = min(B, b0 + per);
  const int64_t page1 = (int64_t(1) << page_shift) - 1;
  const int64_t count = clamped(free_count[0], 0, n_free);

  struct Lengths {
    int64_t ctx, add, extra;
    bool fits;
  };
  // f(b, lengths) for the thread's requests in their order, kBatch loaded at a time.
  auto each = [&](auto f) {
    for (int i = b0; i < b1; i += kBatch) {
      int32_t c[kBatch], n[kBatch];
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        c[e] = ctx_lens[min(i + e, b1 - 1)];
        n[e] = new_lens[min(i + e, b1 - 1)];
      }
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        if (i + e >= b1) break;
        Lengths l;
        l.ctx = max(c[e], 0);
        l.add = max(n[e], 0);
        const int64_t held = (l.ctx + page1) >> page_shift;
        const int64_t need = (l.ctx + l.add + page1) >> page_shift;
        l.fits = need <= width && l.ctx + l.add <= INT32_MAX;
        l.extra = l.fits ? need - held : 0;
        f(i + e, l);
      }
    }
  };

  int64_t ntok = 0, nblk = 0, all_tok, all_blk;
  each([&](int, const Lengths &l) {
    ntok += l.add;
    nblk += l.extra;
  });
  int64_t s = group_exclusive<kThreads>(ntok, part[0], all_tok);
  int64_t f = group_exclusive<kThreads>(nblk, part[1], all_blk);
  // Taken blocks: the requests served form a prefix of those that lack blocks, so
  // their sum is the largest end of one that is served.
  int64_t taken = 0;
  int refused = 0;
  const bool leader = blockIdx.x == 0;
  each([&](int b, const Lengths &l) {
    const bool ok = l.fits && (l.extra == 0 || f + l.extra <= count);
    start[b] = saturated(s);
    first[b] = ok ? saturated(f) : -1;
    if (ok && l.extra > 0) taken = f + l.extra;
    refused += !ok;
    if (leader) {
      query_starts[b] = saturated(s);
      seq_lens[b] = ok ? (int32_t)(l.ctx + l.add) : 0;
    }
    s += l.add;
    f += l.extra;
  });
  if (leader) {
    int64_t served = taken, no = refused;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const int64_t o = __shfl_xor(served, d);
      served = o > served ? o : served;
      no += __shfl_xor(no, d);
    }
    if ((tid & 63) == 0) {
      part[2][tid >> 6] = served;
      part[0][tid >> 6] = no;               // (part[0] was read before the last barrier)
    }
  }
  __syncthreads();
  if (leader && tid == 0) {
    int64_t served = 0, no = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      served = part[2][w] > served ? part[2][w] : served;
      no += part[0][w];
    }
    query_starts[B] = saturated(all_tok);
    counts[0] = (int32_t)(count - served);
    counts[1] = saturated(all_tok);
    counts[2] = (int32_t)no;
  }

  const int64_t t0 = (int64_t)blockIdx.x * kTokensPerGroup;
  for (int i = 0; i < kTokensPerGroup / kThreads; ++i) {
    const int64_t t = t0 + i * kThreads + tid;
    if (t >= tokens) break;
    int32_t slot = -1, pos = 0;
    if (t < all_tok) {
      const int b = owner(start, B, t);
      const int64_t c = max(ctx_lens[b], 0), p = c + (t - start[b]);
      pos = saturated(p);
      if (first[b] >= 0) {
        const int64_t had = (c + page1) >> page_shift, j = p >> page_shift;
        int32_t id;
        if (j < had) {
          id = tables[(int64_t)b * width + j];
        } else {
          id = free_blocks[count - 1 - (first[b] + (j - had))];
          if ((p & page1) == 0) tables[(int64_t)b * width + j] = id;
        }
        // (An entry whose slots int32 does not hold is no block.)
        if (id >= 0 && id <= (INT32_MAX >> page_shift))
          slot = (int32_t)((int64_t)id << page_shift | (p & page1));
      }
    }
    slots[t] = slot;
    positions[t] = pos;
  }
  // Tokens past `tokens` get no slot, but the blocks that begin with them are taken as all
  // others (lengths and counts have them): a wave a request, from the one with token
  // number `tokens` on.
  if (all_tok > tokens) {
    const int waves = kThreads / 64;
    for (int b = owner(start, B, tokens) + (int)blockIdx.x * waves + (tid >> 6); b < B;
         b += (int)gridDim.x * waves) {
      if (first[b] < 0) continue;
      const int64_t c = max(ctx_lens[b], 0), add = max(new_lens[b], 0);
      const int64_t had = (c + page1) >> page_shift, need = (c + add + page1) >> page_shift;
      for (int64_t j = had + (tid & 63); j < need; j += 64)
        if (start[b] + (j << page_shift) - c >= tokens)
          tables[(int64_t)b * width + j] = free_blocks[count - 1 - (first[b] + (j - had))];
    }
  }
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void block_release_kernel(
    const int32_t *__restrict__ lens, const uint8_t *__restrict__ ended, int B,
    const int32_t *__restrict__ tables, int64_t width, int32_t *__restrict__ free_blocks,
    int64_t n_free, const int32_t *__restrict__ free_count, int page_shift,
    int32_t *__restrict__ count_out) {
  extern __shared__ int32_t lds[];          // [B] blocks given back before each request
  __shared__ int64_t part[kThreads / 64];
  const int tid = threadIdx.x, per = (B + kThreads - 1) / kThreads;
  const int b0 = tid * per, b1 = min(B, b0 + per);
  const int64_t page1 = (int64_t(1) << page_shift) - 1;
  const int64_t count = clamped(free_count[0], 0, n_free);
  auto each = [&](auto f) {
    for (int i = b0; i < b1; i += kBatch) {
      int32_t len[kBatch];
      uint8_t end[kBatch];
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        len[e] = lens[min(i + e, b1 - 1)];
        end[e] = ended[min(i + e, b1 - 1)];
      }
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        if (i + e >= b1) break;
        const int64_t n = (max((int64_t)len[e], (int64_t)0) + page1) >> page_shift;
        f(i + e, end[e] ? (n < width ? n : width) : (int64_t)0);
      }
    }
  };
  int64_t n = 0, all;
  each([&](int, int64_t given) { n += given; });
  int64_t f = group_exclusive<kThreads>(n, part, all);
  each([&](int b, int64_t given) {
    lds[b] = saturated(f);
    f += given;
  });
  __syncthreads();
  const int64_t room = n_free - count, copied = all < room ? all : room;
  if (blockIdx.x == 0 && tid == 0) count_out[0] = saturated(count + copied);
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + tid; k < copied; k += step) {
    const int b = owner(lds, B, k);
    free_blocks[count + k] = tables[(int64_t)b * width + (k - lds[b])];
  }
}

int log2_of(int page) { return __builtin_ctz((unsigned)page); }

// f<threads>() for this many requests.
template <class F>
hipError_t with_threads(int B, F f) {
  return B > kFewThreads ? f(std::integral_constant<int, kManyThreads>{})
                         : f(std::integral_constant<int, kFewThreads>{});
}

}  // namespace

hipError_t launch_block_assign(const int32_t *ctx, const int32_t *fresh, int B, int32_t *tables,
                               int64_t width, const int32_t *free_blocks, int64_t n_free,
                               const int32_t *free_count, int page, int64_t tokens,
                               int32_t *slots, int32_t *positions, int32_t *seq_lens,
                               int32_t *query_starts, int32_t *counts, hipStream_t stream) {
  const int64_t groups = (tokens + kTokensPerGroup - 1) / kTokensPerGroup;
  return with_threads(B, [&](auto threads) {
    constexpr int kThreads = decltype(threads)::value;
    static std::atomic<bool> limit[kMaxDevices];
    const auto kernel = block_assign_kernel<kThreads>;
    const hipError_t e = set_lds_limit(limit, (const void *)kernel,
                                       (int)(2 * sizeof(int32_t) * kMaxBlockRequests));
    if (e != hipSuccess) return e;
    kernel<<<(unsigned)(groups > 0 ? groups : 1), kThreads, 2 * sizeof(int32_t) * (B > 0 ? B : 1),
             stream>>>(ctx, fresh, B, tables, width, free_blocks, n_free, free_count,
                       log2_of(page), tokens, slots, positions, seq_lens, query_starts, counts);
    return hipGetLastError();
  });
}

hipError_t launch_block_release(const int32_t *lens, const uint8_t *ended, int B,
                                const int32_t *tables, int64_t width, int32_t *free_blocks,
                                int64_t n_free, const int32_t *free_count, int page,
                                int32_t *count_out, hipStream_t stream) {
  const int64_t entries = B * width < n_free ? B * width : n_free;
  return with_threads(B, [&](auto threads) {
    constexpr int kThreads = decltype(threads)::value;
    static std::atomic<bool> limit[kMaxDevices];
    const auto kernel = block_release_kernel<kThreads>;
    const hipError_t e = set_lds_limit(limit, (const void *)kernel,
                                       (int)(sizeof(int32_t) * kMaxBlockRequests));
    if (e != hipSuccess) return e;
    int64_t groups = (entries + kThreads - 1) / kThreads;
    groups = groups < 1 ? 1 : (groups > 256 ? 256 : groups);
    kernel<<<(unsigned)groups, kThreads, sizeof(int32_t) * (B > 0 ? B : 1), stream>>>(
        lens, ended, B, tables, width, free_blocks, n_free, free_count, log2_of(page), count_out);
    return hipGetLastError();
  });
}

}  // namespace rfq
