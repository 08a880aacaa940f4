// RFQ product with a weight matrix per expert: the slots offsets[e] .. offsets[e + 1] - 1
// are rows of expert e,
//     Z[s][n] = sum_k (deq q + deq r)[rows[s]][k] deq(w_e)[n][k]            (Eq. 11)
// (rows == nullptr: activation row s).  The offsets are read on the device: a launch covers
// the most tiles that P rows of E experts can have, and a workgroup finds its expert by a
// prefix sum over the experts' tiles.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "experts.h"
#include "gemm_common.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void *p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes,
                                           0x00020000);
}

// Workgroups of a launch; each takes every kMostGroups-th tile.
constexpr int kMostGroups = 1 << 20;

// A tile's expert and slots [s0, end): end is the expert's.
struct RowTile { int e, s0, end; };

// Tile t of the experts' row tiles of `rows` slots, in the order of experts; false past the
// last.  Every wave of a workgroup calls it with the same t (all lanes active).
__device__ __forceinline__ bool find_tile(const int32_t *offsets, int E, int P, int rows, int t,
                                          RowTile &tile) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    int b = 0, c = 0;
    if (e < E) {
      b = min(max(offsets[e], 0), P);
      c = min(max(offsets[e + 1], b), P);
    }
    const int tiles = (c - b + rows - 1) / rows;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const uint64_t m = __ballot(before + incl > t);
    if (m) {
      const int l = __builtin_ctzll(m);
      const int at = t - before - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(tiles, l));
      tile.e = e0 + l;
      tile.s0 = __builtin_amdgcn_readlane(b, l) + at * rows;
      tile.end = __builtin_amdgcn_readlane(c, l);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// ---- few rows

constexpr int kFewThreads = 256, kFewWaves = kFewThreads / 64;
constexpr int kFewRows = 16;
constexpr uint32_t kNowhere = 0x80000000u;      // an offset past every buffer: loads zeros

__device__ __forceinline__ v8i frag(const u32x4 &d) {
  return v8i{(int)d.x, (int)d.y, (int)d.z, (int)d.w, 0, 0, 0, 0};
}

// 16 slots of an expert by 16 F of its weight rows a workgroup, whose waves share the
// k-steps of 128 (lane l: row l mod 16, block 4 step + l / 16).
template <bool RES, bool ZBF16, int F>
__global__ __launch_bounds__(kFewThreads) void rfq_gemm_experts_few_kernel(ExpertsGemm a, int ntn,
                                                                           int most) {
  __shared__ v4f partial[kFewWaves][F][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, g = lane >> 4;
  const int64_t kbytes = a.K / 2;
  const int kblocks = (int)(a.K / 32), steps = (kblocks + 3) / 4;
  const int s0 = steps * wave / kFewWaves, s1 = steps * (wave + 1) / kFewWaves;
  // (Never empty, so that a range exceeds every scalar offset: without activations the
  // launch passes weights, and no lane's row is live.)
  const int64_t held = max(a.M, (int64_t)1);
  const __amdgpu_buffer_rsrc_t rq = rsrc(a.qc, held * kbytes), rqs = rsrc(a.qs, held * kblocks),
                               rr = rsrc(RES ? a.rc : a.qc, held * kbytes),
                               rrs = rsrc(RES ? a.rs : a.qs, held * kblocks);
  for (int t = blockIdx.x; t < most; t += gridDim.x) {
    RowTile tile;
    if (!find_tile(a.offsets, a.E, (int)a.P, kFewRows, t / ntn, tile)) return;
    const int n0 = t % ntn * (16 * F);
    const __amdgpu_buffer_rsrc_t rw = rsrc(a.wc + (int64_t)tile.e * a.N * kbytes, a.N * kbytes),
                                 rws = rsrc(a.ws + (int64_t)tile.e * a.N * kblocks, a.N * kblocks);
    const int slot = tile.s0 + row;
    uint32_t m = 0xFFFFFFFFu;
    if (slot < tile.end) m = a.rows ? (uint32_t)a.rows[slot] : (uint32_t)slot;
    const bool live = m < (uint64_t)a.M;
    const uint32_t x_off = live ? m * (uint32_t)kbytes + 16 * g : kNowhere;
    const uint32_t xs_off = live ? m * (uint32_t)kblocks + g : kNowhere;
    uint32_t w_off[F], ws_off[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const bool in = n0 + 16 * f + row < a.N;
      w_off[f] = in ? (uint32_t)(n0 + 16 * f + row) * (uint32_t)kbytes + 16 * g : kNowhere;
      ws_off[f] = in ? (uint32_t)(n0 + 16 * f + row) * (uint32_t)kblocks + g : kNowhere;
    }
    v4f acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = s0; s < s1; ++s) {
      const bool past = 4 * s + g >= kblocks;
      auto code = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off) {
        return __builtin_amdgcn_raw_buffer_load_b128(r, past ? kNowhere : off, 64 * s, 0);
      };
      auto scale = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off) {
        return (int)__builtin_amdgcn_raw_buffer_load_b8(r, past ? kNowhere : off, 4 * s, 0);
      };
      const u32x4 q = code(rq, x_off), r = RES ? code(rr, x_off) : q;
      const int qs = scale(rqs, xs_off), rs = RES ? scale(rrs, xs_off) : 0;
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const u32x4 w = code(rw, w_off[f]);
        const int ws = scale(rws, ws_off[f]);
        acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(w), frag(q), acc[f], kFmtFp4,
                                                                  kFmtFp4, 0, ws, 0, qs);
        if constexpr (RES)
          acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              frag(w), frag(r), acc[f], kFmtFp4, kFmtFp4, 0, ws, 0, rs);
      }
    }
#pragma unroll
    for (int f = 0; f < F; ++f) partial[wave][f][lane] = acc[f];
    __syncthreads();
    for (int f = wave; f < F; f += kFewWaves) {
      v4f s = partial[0][f][lane];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) {
        const v4f p = partial[w][f][lane];
        s = v4f{s[0] + p[0], s[1] + p[1], s[2] + p[2], s[3] + p[3]};
      }
      if (slot < tile.end) {
        const int64_t n = n0 + 16 * f + 4 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (n + i < a.N) {
            const int64_t at = slot * a.N + n + i;
            if constexpr (ZBF16) static_cast<uint16_t *>(a.z)[at] = (uint16_t)bf16_rne(s[i]);
            else static_cast<float *>(a.z)[at] = s[i];
          }
        }
      }
    }
    __syncthreads();
  }
}

}  // namespace

// The few-row tiles, the smallest, are numbered in 32 bits.
bool gemm_experts_fits(int64_t P, int64_t E, int64_t N) {
  const int64_t tiles = std::min<int64_t>(P, P / kFewRows + E), ntn = (N + 15) / 16;
  return tiles == 0 || ntn <= (INT32_MAX - kMostGroups) / tiles;
}

hipError_t launch_gemm_experts(const ExpertsGemm &args, bool z_bf16, hipStream_t stream) {
  ExpertsGemm g = args;
  if (g.M == 0) g.qc = g.wc, g.qs = g.ws, g.rc = nullptr, g.rs = nullptr;
  constexpr int F = 2;
  const int64_t ntn = (g.N + 16 * F - 1) / (16 * F);
  const int64_t tiles = std::min<int64_t>(g.P, g.P / kFewRows + g.E);
  const int64_t most = tiles * ntn;
  auto kern = g.rc ? (z_bf16 ? rfq_gemm_experts_few_kernel<true, true, F>
                             : rfq_gemm_experts_few_kernel<true, false, F>)
                   : (z_bf16 ? rfq_gemm_experts_few_kernel<false, true, F>
                             : rfq_gemm_experts_few_kernel<false, false, F>);
  kern<<<(unsigned)std::min<int64_t>(most, kMostGroups), kFewThreads, 0, stream>>>(g, (int)ntn, (int)most);
  return hipGetLastError();
}

}  // namespace rfq
