// RFQ product with a weight matrix per expert: the slots offsets[e] .. offsets[e + 1] - 1
// are rows of expert e,
//     Z[s][n] = sum_k (deq q + deq r)[rows[s]][k] deq(w_e)[n][k]            (Eq. 11)
// (rows == nullptr: activation row s).  The offsets are read on the device: a launch covers
// the most tiles that P slots of E experts can have, and each workgroup finds its tile by a
// prefix sum over the experts' (experts_device.h).
//
// Experts with few slots are bound by streaming their weights, those with many by the
// matrix cores.  Three launches, by the mean number of slots (P / E; the lengths themselves
// are on the device):
//   few    tiles of 16 slots by 64 weight rows that split K over their waves;
//   both   128 x 128 tiles of the dense product (gemm_tile.h) for the experts with more than
//          kFewSlots slots, and in the same launch few-row tiles for the others;
//   many   256 x 256 tiles of the dense product, whose waves idle past an expert's end.
// Measured (us, with the residual; T tokens choose 8 of 128 experts, weights 1536 x 2048 each,
// bf16 Z):          T =   16    64   128   512  1024  2048  4096
//                  few  33.6  53.0  69.3   124   145     -     -
//                 both  32.8  49.8  56.0  68.9  80.3   113   188
//                 many  38.1  58.2  60.7  71.6  88.5   106   157
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
constexpr int kFewRows = 16;                    // slots of a tile
constexpr uint32_t kNowhere = 0x80000000u;      // an offset past every buffer: loads zeros

// 16 slots of an expert by 64 of its weight rows (four fragments) a workgroup, whose four
// waves share the k-steps of 128 (v_mfma_scale_f32_16x16x128_f8f6f4, lane l: row l mod 16,
// block 4 step + l / 16 of its operand; weights are the first operand, so that a lane gets four
// consecutive outputs of a row) and add their results through LDS in a fixed order.  The loads
// of U steps are issued together, those of the next U weights before the products.  Scale
// bytes are loaded one a lane, so that a row's may start anywhere.
//
// Bound by the weights' way from memory: 8 experts of 12288 x 2048 (107 MB) with two slots each
// 32 us, where a maximum over as many bytes takes 25.5.  Two, four or eight fragments, U from
// one to four and non-temporal loads are within 5% of that or slower; up to K = 1536, where a
// wave has at most three steps, U = 1 (64 tokens, 128 experts of 2048 x 768: 26.5 -> 23.5).
constexpr int kFrags = 4, kFewCols = 16 * kFrags;
constexpr int kFewBytes = kFewWaves * kFrags * 64 * 16;
constexpr int64_t kShortK = 1536;

template <bool RES, bool ZBF16, int U>
__device__ __forceinline__ void few_tile(const ExpertsGemm &a, const ExpertTiles &ex, int bid,
                                         v4f (*partial)[kFrags][64]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, g = lane >> 4;
  const int64_t kbytes = a.K / 2;
  const int kblocks = (int)(a.K / 32), steps = (kblocks + 3) / 4;
  const int s0 = steps * wave / kFewWaves, s1 = steps * (wave + 1) / kFewWaves;
  RowTile tile;
  if (!expert_tile<kFewRows, 64, false>(ex, bid, (int)((a.N + kFewCols - 1) / kFewCols), tile))
    return;
  const int n0 = tile.tn * kFewCols;
  auto rsrc = [](const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t rq = rsrc(a.qc, a.M * kbytes), rqs = rsrc(a.qs, a.M * kblocks),
                               rr = rsrc(RES ? a.rc : a.qc, a.M * kbytes),
                               rrs = rsrc(RES ? a.rs : a.qs, a.M * kblocks),
                               rw = rsrc(a.wc + (int64_t)tile.e * a.N * kbytes, a.N * kbytes),
                               rws = rsrc(a.ws + (int64_t)tile.e * a.N * kblocks, a.N * kblocks);
  // Step s + u of an operand; steps past the wave's last, and blocks past K, load zeros.
  auto code = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int s, int u) {
    const bool past = s + u >= s1 || 4 * (s + u) + g >= kblocks;
    return __builtin_amdgcn_raw_buffer_load_b128(r, past ? kNowhere : off + 64 * u, 64 * s, 0);
  };
  auto scale = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int s, int u) {
    const bool past = s + u >= s1 || 4 * (s + u) + g >= kblocks;
    return (int)__builtin_amdgcn_raw_buffer_load_b8(r, past ? kNowhere : off + 4 * u, 4 * s, 0);
  };
  uint32_t w_off[kFrags], ws_off[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    const int n = n0 + 16 * f + row;
    w_off[f] = n < a.N ? (uint32_t)n * (uint32_t)kbytes + 16 * g : kNowhere;
    ws_off[f] = n < a.N ? (uint32_t)n * (uint32_t)kblocks + g : kNowhere;
  }
  struct Weights { u32x4 c[kFrags][U]; int s[kFrags][U]; };
  auto load_w = [&](Weights &w, int s) {
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w.c[f][u] = code(rw, w_off[f], s, u);
        w.s[f][u] = scale(rws, ws_off[f], s, u);
      }
  };
  Weights w0, w1;
  load_w(w0, s0);          // (Before the row indices, which the activations wait for.)
  __builtin_amdgcn_sched_barrier(0);
  const int slot = tile.s0 + row;
  const uint32_t m = slot < tile.end ? expert_row(ex, slot) : 0xFFFFFFFFu;
  const bool live = m < a.M;
  const uint32_t x_off = live ? m * (uint32_t)kbytes + 16 * g : kNowhere;
  const uint32_t xs_off = live ? m * (uint32_t)kblocks + g : kNowhere;
  v4f acc[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) acc[f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // U steps: the activations, the next weights, the products.
  auto multiply = [&](const Weights &w, Weights &next, int s) {
    u32x4 q[U], r[RES ? U : 1];
    int qsc[U], rsc[RES ? U : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      q[u] = code(rq, x_off, s, u);
      qsc[u] = scale(rqs, xs_off, s, u);
      if constexpr (RES) {
        r[u] = code(rr, x_off, s, u);
        rsc[u] = scale(rrs, xs_off, s, u);
      }
    }
    if (s + U < s1) load_w(next, s + U);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            as_v8i(w.c[f][u]), as_v8i(q[u]), acc[f], kFmtFp4, kFmtFp4, 0, w.s[f][u], 0, qsc[u]);
        if constexpr (RES)
          acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              as_v8i(w.c[f][u]), as_v8i(r[u]), acc[f], kFmtFp4, kFmtFp4, 0, w.s[f][u], 0, rsc[u]);
      }
  };
  for (int s = s0; s < s1; s += 2 * U) {
    multiply(w0, w1, s);
    if (s + U < s1) multiply(w1, w0, s + U);
  }
#pragma unroll
  for (int f = 0; f < kFrags; ++f) partial[wave][f][lane] = acc[f];
  __syncthreads();
  // Wave f adds and stores fragment f.
  static_assert(kFrags == kFewWaves, "a fragment a wave");
  v4f s = partial[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kFewWaves; ++w) {
    const v4f p = partial[w][wave][lane];
    s = v4f{s[0] + p[0], s[1] + p[1], s[2] + p[2], s[3] + p[3]};
  }
  const int64_t n = n0 + 16 * wave + 4 * g;
  if (slot >= tile.end || n >= a.N) return;
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

template <bool RES, bool ZBF16, int U>
__global__ __launch_bounds__(kFewThreads) void rfq_gemm_experts_few_kernel(ExpertsGemm a,
                                                                           ExpertTiles ex) {
  __shared__ v4f partial[kFewWaves][kFrags][64];
  few_tile<RES, ZBF16, U>(a, ex, (int)blockIdx.x, partial);
}

// ---- many rows

template <class C, bool RES, bool ZBF16, bool GK>
__device__ __forceinline__ void multiply_tile(const ExpertsGemm &a, const ExpertTiles &ex,
                                              const RowTile &tile) {
  auto go = [&](auto idle) {
    gemm_tile<C, RES, ZBF16, false, false, false, false, GK, true, decltype(idle)::value>(
        a.qc, a.qs, a.rc, a.rs, a.wc, a.ws, a.M, a.N, a.K, a.z, SwigluOut{}, nullptr, a.K, ex, tile);
  };
  if (__builtin_amdgcn_readfirstlane(tile.s0 + expert_wave_row<C>() * C::kTM < tile.end))
    go(std::false_type{});
  else
    go(std::true_type{});
}

// A tile of C; with S another shape of the same columns, that one where it holds the rest of
// the expert.
template <class C, class S, bool RES, bool ZBF16, bool GK>
__device__ __forceinline__ void many_tile(const ExpertsGemm &a, const ExpertTiles &ex) {
  static_assert(C::kBN == S::kBN && C::kThreads == S::kThreads, "the same columns and waves");
  RowTile tile;
  if (!expert_tile<C::kBM, 1024 / C::kBM, true>(ex, (int)blockIdx.x,
                                                (int)((a.N + C::kBN - 1) / C::kBN), tile))
    return;
  if constexpr (!std::is_same<C, S>::value) {
    if (tile.end - tile.s0 <= S::kBM) return multiply_tile<S, RES, ZBF16, GK>(a, ex, tile);
  }
  multiply_tile<C, RES, ZBF16, GK>(a, ex, tile);
}

template <bool RES, bool ZBF16, bool GK>
__global__ __launch_bounds__(Big::kThreads, 2) void rfq_gemm_experts_many_kernel(ExpertsGemm a,
                                                                                 ExpertTiles ex) {
  many_tile<Big, Half, RES, ZBF16, GK>(a, ex);
}

// The first `tiles` workgroups take the experts with many slots, the others those with few,
// whose weights stream while the former keep the matrix cores busy (two launches: 701 tokens,
// 60 experts of 2048 x 1408, plain: 41 us, 33 in one).
template <bool RES, bool ZBF16, bool GK>
__global__ __launch_bounds__(Mid::kThreads, 3) void rfq_gemm_experts_both_kernel(
    ExpertsGemm a, ExpertTiles many, ExpertTiles few, int tiles) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  if ((int)blockIdx.x < tiles)
    many_tile<Mid, Mid, RES, ZBF16, GK>(a, many);
  else
    few_tile<RES, ZBF16, 2>(a, few, (int)blockIdx.x - tiles,
                            reinterpret_cast<v4f(*)[kFrags][64]>(smem));
}
static_assert(Mid::kThreads == kFewThreads, "one launch for both");

// ---- launches (tiles in eighths: the XCDs')

int64_t few_tiles(int64_t slots_tiles, int64_t N) {
  return (slots_tiles * ((N + kFewCols - 1) / kFewCols) + 7) / 8 * 8;
}
template <class C>
int64_t many_tiles(int64_t P, int64_t experts, int64_t N) {
  return ((P / C::kBM + experts) * ((N + C::kBN - 1) / C::kBN) + 7) / 8 * 8;
}
template <class C, bool RES, bool ZBF16>
constexpr int lds_bytes() {
  constexpr int kEpi = (C::kThreads / 64) * Epi<ZBF16>::kWaveBytes;
  return Layout<C, RES>::kBytes > kEpi ? Layout<C, RES>::kBytes : kEpi;
}

template <bool RES, bool ZBF16, int U>
hipError_t launch_few(const ExpertsGemm &g, const ExpertTiles &ex, hipStream_t stream) {
  const int64_t tiles = few_tiles(std::min<int64_t>(g.P, g.P / kFewRows + g.E), g.N);
  rfq_gemm_experts_few_kernel<RES, ZBF16, U><<<(unsigned)tiles, kFewThreads, 0, stream>>>(g, ex);
  return hipGetLastError();
}

template <bool RES, bool ZBF16, bool GK>
hipError_t launch_both(const ExpertsGemm &g, const ExpertTiles &ex, int few_slots,
                       hipStream_t stream) {
  constexpr int kMid = lds_bytes<Mid, RES, ZBF16>(), kBytes = kMid > kFewBytes ? kMid : kFewBytes;
  auto kern = rfq_gemm_experts_both_kernel<RES, ZBF16, GK>;
  static std::atomic<bool> attr_done[kMaxDevices];
  const hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), kBytes);
  if (e != hipSuccess) return e;
  ExpertTiles many = ex, few = ex;
  many.above = few.most = few_slots;
  // At most P / (few_slots + 1) experts have more than few_slots slots; an expert with fewer
  // has one tile.
  const int64_t tiles = many_tiles<Mid>(g.P, std::min<int64_t>(g.E, g.P / (few_slots + 1)), g.N);
  const int64_t rest = few_tiles(std::min<int64_t>(g.P, g.E), g.N);
  kern<<<(unsigned)(tiles + rest), Mid::kThreads, kBytes, stream>>>(g, many, few, (int)tiles);
  return hipGetLastError();
}

template <bool RES, bool ZBF16, bool GK>
hipError_t launch_many(const ExpertsGemm &g, const ExpertTiles &ex, hipStream_t stream) {
  constexpr int kBytes = lds_bytes<Big, RES, ZBF16>();
  auto kern = rfq_gemm_experts_many_kernel<RES, ZBF16, GK>;
  static std::atomic<bool> attr_done[kMaxDevices];
  const hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), kBytes);
  if (e != hipSuccess) return e;
  const int64_t tiles = many_tiles<Big>(g.P, std::min<int64_t>(g.E, g.P), g.N);
  kern<<<(unsigned)tiles, Big::kThreads, kBytes, stream>>>(g, ex);
  return hipGetLastError();
}

// Few-row tiles alone up to four slots an expert (128 experts of 2048 x 768, 64 tokens: few
// 23.5 us, both 26.5, at 128 tokens 33.9 and 32.5; 8 experts of 4096 x 4096, 16 tokens 21.4 and
// 26.3), as long as a single expert that has all of them costs little.
bool use_few(const ExpertsGemm &g) { return g.P <= 4 * (int64_t)g.E && g.P <= 1024; }
// 256 x 256 tiles from 96 slots an expert where 128 x 128 ones would number two a CU (8 experts
// of 4096 x 4096: 256 slots each 51.6 us, both 62; 128 each, 384 tiles, 46 and 38).
bool use_many(const ExpertsGemm &g) {
  return g.P >= 96 * (int64_t)g.E && (g.P / 128 + g.E / 2) * ((g.N + 127) / 128) >= 512;
}
// Slots up to which an expert runs few-row tiles in a launch of both: 8, or 16 where a 128 x 128
// tile has so few stages that it costs more than the weights it saves (60 experts of
// 2048 x 1408, 512 tokens of 4 choices: 38.6 us with 8, 33.8 with 16; 8 experts of
// 4096 x 4096, 64 tokens of 2: 24.7 and 29.5).
constexpr int kFewSlots = 8, kFewSlotsShortK = 16;
static_assert(kFewSlotsShortK <= kFewRows, "one few-row tile an expert");

}  // namespace

// The tiles of any of the launches, in work items.
bool gemm_experts_fits(int64_t P, int64_t E, int64_t N) {
  return (P / 128 + 2 * E) == 0 || (N + 63) / 64 <= ((1 << 24) - 16) / (P / 128 + 2 * E);
}

hipError_t launch_gemm_experts(const ExpertsGemm &g, bool z_bf16, hipStream_t stream) {
  const ExpertTiles ex{g.offsets, g.rows, g.E, (int)g.P, 0, INT32_MAX};
  const bool short_k = g.K <= kShortK, gk = g.K % (kStageK * kGroup) != 0;
  auto go = [&](auto res, auto zb) {
    constexpr bool R = decltype(res)::value, Z = decltype(zb)::value;
    if (use_few(g))
      return short_k ? launch_few<R, Z, 1>(g, ex, stream) : launch_few<R, Z, 2>(g, ex, stream);
    if (use_many(g))
      return gk ? launch_many<R, Z, true>(g, ex, stream) : launch_many<R, Z, false>(g, ex, stream);
    const int few = short_k ? kFewSlotsShortK : kFewSlots;
    return gk ? launch_both<R, Z, true>(g, ex, few, stream)
              : launch_both<R, Z, false>(g, ex, few, stream);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (g.rc) return z_bf16 ? go(Yes{}, Yes{}) : go(Yes{}, No{});
  return z_bf16 ? go(No{}, Yes{}) : go(No{}, No{});
}

}  // namespace rfq
