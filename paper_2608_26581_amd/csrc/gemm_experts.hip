// RFQ product with a weight matrix per expert: the slots offsets[e] .. offsets[e + 1] - 1
// are rows of expert e,
//     Z[s][n] = sum_k (deq q + deq r)[rows[s]][k] deq(w_e)[n][k]            (Eq. 11)
// (rows == nullptr: activation row s).  The offsets are read on the device: a launch covers
// the most tiles that P slots of E experts can have, and each workgroup finds its tile by a
// prefix sum over the experts' (experts_device.h).
//
// Experts with few slots are bound by streaming their weights, those with many by the
// matrix cores; one launch takes the former with the few-row tiles below, another the
// latter with the tiles of the dense product (gemm_tile.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "experts.h"
#include "gemm_tile.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

// ---- few rows

constexpr int kFewThreads = 256, kFewWaves = kFewThreads / 64;
constexpr uint32_t kNowhere = 0x80000000u;      // an offset past every buffer: loads zeros

// 16 S slots of an expert by 16 F of its weight rows a workgroup, whose four waves share the
// k-steps of 128 (v_mfma_scale_f32_16x16x128_f8f6f4, lane l: row l mod 16, block
// 4 step + l / 16 of its operand; weights are the first operand, so that a lane gets four
// consecutive outputs of a row) and add their results through LDS in a fixed order.  U
// steps' loads are issued together.  Scale bytes are loaded one a lane, so that a row's may
// start anywhere.
template <bool RES, bool ZBF16, int S, int F, int U>
__global__ __launch_bounds__(kFewThreads) void rfq_gemm_experts_few_kernel(ExpertsGemm a,
                                                                           ExpertTiles ex) {
  __shared__ v4f partial[kFewWaves][S * F][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, g = lane >> 4;
  const int64_t kbytes = a.K / 2;
  const int kblocks = (int)(a.K / 32), steps = (kblocks + 3) / 4;
  const int s0 = steps * wave / kFewWaves, s1 = steps * (wave + 1) / kFewWaves;
  RowTile tile;
  int tn;
  if (!expert_tile<16 * S, 1024>(ex, (int)((a.N + 16 * F - 1) / (16 * F)), tile, tn)) return;
  const int n0 = tn * (16 * F);
  auto rsrc = [](const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
  };
  // (Never empty, so that a range exceeds every scalar offset: without activations the
  // launch passes weights, and no lane's row is live.)
  const int64_t held = max(a.M, (int64_t)1);
  const __amdgpu_buffer_rsrc_t rq = rsrc(a.qc, held * kbytes), rqs = rsrc(a.qs, held * kblocks),
                               rr = rsrc(RES ? a.rc : a.qc, held * kbytes),
                               rrs = rsrc(RES ? a.rs : a.qs, held * kblocks),
                               rw = rsrc(a.wc + (int64_t)tile.e * a.N * kbytes, a.N * kbytes),
                               rws = rsrc(a.ws + (int64_t)tile.e * a.N * kblocks, a.N * kblocks);
  const int slices = min(S, (tile.end - tile.s0 + 15) / 16);
  uint32_t x_off[S], xs_off[S], w_off[F], ws_off[F];
#pragma unroll
  for (int sl = 0; sl < S; ++sl) {
    const int slot = tile.s0 + 16 * sl + row;
    const uint32_t m = slot < tile.end ? expert_row(ex, slot) : 0xFFFFFFFFu;
    const bool live = m < a.M;
    x_off[sl] = live ? m * (uint32_t)kbytes + 16 * g : kNowhere;
    xs_off[sl] = live ? m * (uint32_t)kblocks + g : kNowhere;
  }
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const int n = n0 + 16 * f + row;
    w_off[f] = n < a.N ? (uint32_t)n * (uint32_t)kbytes + 16 * g : kNowhere;
    ws_off[f] = n < a.N ? (uint32_t)n * (uint32_t)kblocks + g : kNowhere;
  }
  v4f acc[S][F];
#pragma unroll
  for (int sl = 0; sl < S; ++sl)
#pragma unroll
    for (int f = 0; f < F; ++f) acc[sl][f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = s0; s < s1; s += U) {
    // (Steps past the wave's last, and blocks past K, load zeros.)
    auto code = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int u) {
      const bool past = s + u >= s1 || 4 * (s + u) + g >= kblocks;
      return __builtin_amdgcn_raw_buffer_load_b128(r, past ? kNowhere : off, 64 * s, 0);
    };
    auto scale = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int u) {
      const bool past = s + u >= s1 || 4 * (s + u) + g >= kblocks;
      return (int)__builtin_amdgcn_raw_buffer_load_b8(r, past ? kNowhere : off, 4 * s, 0);
    };
    u32x4 w[F][U];
    int wsc[F][U];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[f][u] = code(rw, w_off[f] + 64 * u, u);
        wsc[f][u] = scale(rws, ws_off[f] + 4 * u, u);
      }
#pragma unroll
    for (int sl = 0; sl < S; ++sl) {
      if (sl >= slices) break;
      u32x4 q[U], r[RES ? U : 1];
      int qsc[U], rsc[RES ? U : 1];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        q[u] = code(rq, x_off[sl] + 64 * u, u);
        qsc[u] = scale(rqs, xs_off[sl] + 4 * u, u);
        if constexpr (RES) {
          r[u] = code(rr, x_off[sl] + 64 * u, u);
          rsc[u] = scale(rrs, xs_off[sl] + 4 * u, u);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          acc[sl][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              as_v8i(w[f][u]), as_v8i(q[u]), acc[sl][f], kFmtFp4, kFmtFp4, 0, wsc[f][u], 0, qsc[u]);
          if constexpr (RES)
            acc[sl][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                as_v8i(w[f][u]), as_v8i(r[u]), acc[sl][f], kFmtFp4, kFmtFp4, 0, wsc[f][u], 0, rsc[u]);
        }
    }
  }
#pragma unroll
  for (int sl = 0; sl < S; ++sl)
#pragma unroll
    for (int f = 0; f < F; ++f) partial[wave][sl * F + f][lane] = acc[sl][f];
  __syncthreads();
  for (int p = wave; p < slices * F; p += kFewWaves) {
    v4f s = partial[0][p][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) {
      const v4f q = partial[w][p][lane];
      s = v4f{s[0] + q[0], s[1] + q[1], s[2] + q[2], s[3] + q[3]};
    }
    const int slot = tile.s0 + 16 * (p / F) + row;
    const int64_t n = n0 + 16 * (p % F) + 4 * g;
    if (slot >= tile.end || n >= a.N) continue;
    const int64_t at = slot * a.N + n;
    if constexpr (ZBF16) {
      uint16_t *z = static_cast<uint16_t *>(a.z) + at;
      const uint2 v = make_uint2(bf16x2_rne(s[0], s[1]), bf16x2_rne(s[2], s[3]));
      if (a.N % 4 == 0) {
        *reinterpret_cast<uint2 *>(z) = v;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < a.N) z[i] = (uint16_t)((i < 2 ? v.x : v.y) >> (16 * (i & 1)));
      }
    } else {
      float *z = static_cast<float *>(a.z) + at;
      if (a.N % 4 == 0) {
        *reinterpret_cast<v4f *>(z) = s;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < a.N) z[i] = s[i];
      }
    }
  }
}

template <int S, int F, int U>
hipError_t launch_few(const ExpertsGemm &g, const ExpertTiles &ex, bool z_bf16, hipStream_t stream) {
  const int64_t ntn = (g.N + 16 * F - 1) / (16 * F);
  const int64_t tiles = (std::min<int64_t>(g.P, g.P / (16 * S) + g.E) * ntn + 7) / 8 * 8;
  auto kern = g.rc ? (z_bf16 ? rfq_gemm_experts_few_kernel<true, true, S, F, U>
                             : rfq_gemm_experts_few_kernel<true, false, S, F, U>)
                   : (z_bf16 ? rfq_gemm_experts_few_kernel<false, true, S, F, U>
                             : rfq_gemm_experts_few_kernel<false, false, S, F, U>);
  kern<<<(unsigned)tiles, kFewThreads, 0, stream>>>(g, ex);
  return hipGetLastError();
}

// ---- many rows

template <class C, bool RES, bool ZBF16, bool GK>
__global__ __launch_bounds__(C::kThreads, C::kThreads > 256 || C::kDepth > 1 ? 2 : 3) void
rfq_gemm_experts_tile_kernel(ExpertsGemm a, ExpertTiles ex) {
  gemm_tile<C, RES, ZBF16, false, false, false, false, GK, true>(
      a.qc, a.qs, a.rc, a.rs, a.wc, a.ws, a.M, a.N, a.K, a.z, SwigluOut{}, nullptr, a.K, ex);
}

template <class C, bool RES, bool ZBF16, bool GK>
hipError_t launch_tiles(const ExpertsGemm &g, const ExpertTiles &ex, hipStream_t stream) {
  using L = Layout<C, RES>;
  constexpr int kEpiBytes = (C::kThreads / 64) * Epi<ZBF16>::kWaveBytes;
  constexpr int kBytes = L::kBytes > kEpiBytes ? L::kBytes : kEpiBytes;
  auto kern = rfq_gemm_experts_tile_kernel<C, RES, ZBF16, GK>;
  static std::atomic<bool> attr_done[kMaxDevices];
  const hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), kBytes);
  if (e != hipSuccess) return e;
  // Experts with more than `above` slots: at most P / (above + 1) of them.
  const int64_t experts = std::min<int64_t>(g.E, g.P / (ex.above + 1));
  const int64_t ntn = (g.N + C::kBN - 1) / C::kBN;
  const int64_t tiles = ((g.P / C::kBM + experts) * ntn + 7) / 8 * 8;
  if (experts == 0) return hipSuccess;
  kern<<<(unsigned)tiles, C::kThreads, kBytes, stream>>>(g, ex);
  return hipGetLastError();
}

template <class C>
hipError_t launch_tiles(const ExpertsGemm &g, const ExpertTiles &ex, bool z_bf16,
                        hipStream_t stream) {
  auto go = [&](auto res, auto zb) {
    constexpr bool R = decltype(res)::value, Z = decltype(zb)::value;
    return g.K % (kStageK * kGroup) ? launch_tiles<C, R, Z, true>(g, ex, stream)
                                    : launch_tiles<C, R, Z, false>(g, ex, stream);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (g.rc) return z_bf16 ? go(Yes{}, Yes{}) : go(Yes{}, No{});
  return z_bf16 ? go(No{}, Yes{}) : go(No{}, No{});
}

}  // namespace

// A launch's work items: the few-row tiles, 16 slots by 32 weight rows, are the smallest.
bool gemm_experts_fits(int64_t P, int64_t E, int64_t N) {
  const int64_t tiles = std::min<int64_t>(P, P / 16 + E), ntn = (N + 31) / 32;
  return tiles == 0 || ntn <= (UINT32_MAX / kFewThreads - 8) / tiles;
}

hipError_t launch_gemm_experts(const ExpertsGemm &args, bool z_bf16, hipStream_t stream) {
  ExpertsGemm g = args;
  if (g.M == 0) g.qc = g.wc, g.qs = g.ws, g.rc = nullptr, g.rs = nullptr;
  constexpr int kFewSlots = 64;
  ExpertTiles ex{g.offsets, g.rows, g.E, (int)g.P, 0, INT32_MAX};
  const bool many = g.M > 0 && g.P > 512, few = !many || g.P < 128 * (int64_t)g.E;
  if (few) {
    if (many) ex.most = kFewSlots;
    const hipError_t e = g.P <= 8 * (int64_t)g.E    ? launch_few<1, 2, 4>(g, ex, z_bf16, stream)
                         : g.P <= 24 * (int64_t)g.E ? launch_few<2, 2, 4>(g, ex, z_bf16, stream)
                                                    : launch_few<4, 2, 4>(g, ex, z_bf16, stream);
    if (e != hipSuccess || !many) return e;
    ex.above = kFewSlots;
    ex.most = INT32_MAX;
  }
  return launch_tiles<Mid>(g, ex, z_bf16, stream);
}

}  // namespace rfq
