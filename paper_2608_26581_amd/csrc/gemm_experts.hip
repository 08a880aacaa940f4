// RFQ product with a weight matrix per expert: the slots offsets[e] .. offsets[e + 1] - 1
// are rows of expert e,
//     Z[s][n] = sum_k (deq q + deq r)[rows[s]][k] deq(w_e)[n][k]            (Eq. 11)
// (rows == nullptr: activation row s).  The offsets are read on the device: a launch covers
// the most tiles that P slots of E experts can have, and each workgroup finds its tile by a
// prefix sum over the experts' (experts_device.h).
//
// Experts with few slots are bound by streaming their weights, those with many by the
// matrix cores.  Two launches, by P / E, the mean number of slots where every pair's expert is
// held here (the lengths themselves are on the device; use_many()):
//   both   128 x 128 tiles of the dense product (gemm_tile.h) for the experts with more than
//          16 slots, and in the same launch tiles of 16 slots by 64 weight rows for the others;
//   many   256 x 256 tiles of the dense product, or 128 x 256 at an expert's end.
// Measured (us, with the residual; T tokens choose 8 of 128 experts, weights 1536 x 2048 each,
// bf16 Z):          T =   16    64   128   512  1024  2048  4096
//                 both  26.0  41.9  48.2  64.1  80.3   113   188
//                 many  38.1  58.2  60.7  71.6  88.5   106   157
// With experts of equal length the product takes the dense product's time: 32768 x 1536 x 2048
// 106 us for 64 experts, 118 dense.
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
// consecutive outputs of a row) and add their results through LDS in a fixed order.  A wave
// loads kSteps steps, multiplies them and loads the next: a second set of registers leaves too
// few waves on a SIMD (decode of 16 tokens, 128 experts of 1536 x 2048: 26 us, 30 with it; four
// steps at once 29).
//
// The scale bytes of up to kFewK columns come through LDS.  Loaded a byte a lane next to the
// codes, as rows that start anywhere call for, they took as many requests as the codes: 33 us,
// 23 without them.  FAST (K a multiple of 128 and at most kFewK): those of 64 weight rows are
// one run of memory, which the workgroup copies 16 bytes a lane, and those of q and r whole
// dwords.
//
// Other K stage their scale bytes in pieces of kFewK columns, whole dwords where K is a
// multiple of 128, else byte by byte.  Decode of 16 tokens that choose 68 of 128 experts of 1536
// rows, us: K = 2048 26.2 (staged in pieces 32.4), 4096 44.3 (57.6); in pieces 4224 66.4, 5120 74.2,
// 7168 97.3, byte by byte 2080 57.2.  With kFewK = 8192, whose scale bytes take twice the
// registers, 2048 and 4096 take 26.6 and 44.6, and 4224, 5120 and 7168 49.6, 59.0 and 72.5.
constexpr int kFrags = 4, kFewCols = 16 * kFrags;
constexpr int kSteps = 2, kFewK = 4096, kFewBlocks = kFewK / 32;

// LDS of a few-row tile: scale bytes of weight rows (and 16 before them), of q and of r, [row]
// [block]; then the waves' results.
__host__ __device__ constexpr int few_lds_blocks(int64_t K) {
  return (int)((K < kFewK ? K : kFewK) / 32);
}
__host__ __device__ constexpr int few_lds_bytes(int64_t K) {
  const int scales = 16 + (kFewCols + 2 * kFewRows) * few_lds_blocks(K);
  constexpr int kSums = kFewWaves * kFrags * 64 * 16;
  return scales > kSums ? scales : kSums;
}

template <bool RES, bool ZBF16, bool FAST>
__device__ __forceinline__ void few_tile(const ExpertsGemm &a, const ExpertTiles &ex, int bid,
                                         uint8_t *lds) {
  constexpr int U = kSteps;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, g = lane >> 4;
  const int64_t kbytes = a.K / 2;
  const int kblocks = (int)(a.K / 32), steps = (kblocks + 3) / 4;
  RowTile tile;
  if (!expert_tile<kFewRows, 64, false>(ex, bid, (int)((a.N + kFewCols - 1) / kFewCols), tile))
    return;
  const int n0 = tile.tn * kFewCols;
  auto rsrc = [](const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
  };
  // (Scale ranges end at a whole dword: the tensors start at 16 bytes.)
  auto whole = [](int64_t bytes) { return (bytes + 3) / 4 * 4; };
  const uint8_t *ws = a.ws + ((int64_t)tile.e * a.N + n0) * kblocks;
  const int ws_rem = (int)(reinterpret_cast<uintptr_t>(ws) & 15);
  const __amdgpu_buffer_rsrc_t rq = rsrc(a.qc, a.M * kbytes), rqs = rsrc(a.qs, whole(a.M * kblocks)),
                               rr = rsrc(RES ? a.rc : a.qc, a.M * kbytes),
                               rrs = rsrc(RES ? a.rs : a.qs, whole(a.M * kblocks)),
                               rw = rsrc(a.wc + (int64_t)tile.e * a.N * kbytes, a.N * kbytes),
                               rws = rsrc(ws - ws_rem, whole(ws_rem + (a.N - n0) * kblocks));
  const int slot = tile.s0 + row;
  const uint32_t m = slot < tile.end ? expert_row(ex, slot) : 0xFFFFFFFFu;

  // Scale bytes of a chunk: blocks cb .. cb + nb - 1 of a row at wl (ql, rl) + row * stride.
  const int stride = FAST ? kblocks : min(kblocks, kFewBlocks);
  uint8_t *const wl = lds + (FAST ? ws_rem : 0), *const ql = lds + 16 + kFewCols * stride,
          *const rl = ql + kFewRows * stride;
  // The start of q's or r's scale bytes of tile row `at`, which is lane `at`'s (all lanes call).
  auto x_start = [&](int at) {
    const uint32_t i = (uint32_t)__shfl((int)m, at);
    return i < a.M ? i * (uint32_t)kblocks : kNowhere;
  };
  // nb scale bytes from block cb on of `rows` rows, which start at off(row) of a buffer
  // (kNowhere: zeros), into LDS; whole dwords where K is a multiple of 128.
  auto stage = [&](const __amdgpu_buffer_rsrc_t &r, uint8_t *to, int rows, int cb, int nb, auto off) {
    const int unit = kblocks % 4 == 0 ? 4 : 1, per = nb / unit, total = rows * per;
    for (int i0 = 0; i0 < total; i0 += kFewThreads) {
      const int i = i0 + tid, at = min(i / per, rows - 1), d = unit * (i - at * per);
      const uint32_t o = off(at), from = i < total && o != kNowhere ? o + cb + d : kNowhere;
      if (unit == 4) {
        const uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(r, from, 0, 0);
        if (i < total) *reinterpret_cast<uint32_t *>(to + at * stride + d) = v;
      } else {
        const uint8_t v = __builtin_amdgcn_raw_buffer_load_b8(r, from, 0, 0);
        if (i < total) to[at * stride + d] = v;
      }
    }
  };

  const bool live = m < a.M;
  const uint32_t x_off = live ? m * (uint32_t)kbytes + 16 * g : kNowhere;
  uint32_t w_off[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    const int n = n0 + 16 * f + row;
    w_off[f] = n < a.N ? (uint32_t)n * (uint32_t)kbytes + 16 * g : kNowhere;
  }
  v4f acc[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) acc[f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  struct Codes { u32x4 w[kFrags][U], q[U], r[RES ? U : 1]; };
  for (int c0 = 0; c0 < (FAST ? 1 : steps); c0 += kFewBlocks / 4) {
    const int c1 = FAST ? steps : min(steps, c0 + kFewBlocks / 4), cb = 4 * c0;
    const int s0 = c0 + (c1 - c0) * wave / kFewWaves, s1 = c0 + (c1 - c0) * (wave + 1) / kFewWaves;
    // Steps past the wave's last, and blocks past K, load zeros.
    auto past = [&](int s) { return s >= s1 || (!FAST && 4 * s + g >= kblocks); };
    auto code = [&](const __amdgpu_buffer_rsrc_t &r, uint32_t off, int s, int u) {
      return __builtin_amdgcn_raw_buffer_load_b128(r, past(s + u) ? kNowhere : off + 64 * u, 64 * s, 0);
    };
    auto load_w = [&](Codes &b, int s) {
#pragma unroll
      for (int f = 0; f < kFrags; ++f)
#pragma unroll
        for (int u = 0; u < U; ++u) b.w[f][u] = code(rw, w_off[f], s, u);
    };
    auto load_x = [&](Codes &b, int s) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        b.q[u] = code(rq, x_off, s, u);
        if constexpr (RES) b.r[u] = code(rr, x_off, s, u);
      }
    };
    auto multiply = [&](const Codes &b, int s) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool none = past(s + u);
        const int at = none ? 0 : 4 * (s + u) + g - cb;
        auto scale = [&](const uint8_t *p, int r) { return none ? 0 : (int)p[r * stride + at]; };
        const int qs = scale(ql, row), rs = RES ? scale(rl, row) : 0;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          const int wsc = scale(wl, 16 * f + row);
          acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              as_v8i(b.w[f][u]), as_v8i(b.q[u]), acc[f], kFmtFp4, kFmtFp4, 0, wsc, 0, qs);
          if constexpr (RES)
            acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                as_v8i(b.w[f][u]), as_v8i(b.r[u]), acc[f], kFmtFp4, kFmtFp4, 0, wsc, 0, rs);
        }
      }
    };
    if (c0 > 0) __syncthreads();         // (The chunk before is read.)
    Codes b0;
    if constexpr (FAST) {
      // All loads before the first is waited for, the weights' scales first.
      constexpr int kW = kFewCols * kFewBlocks / 16 / kFewThreads,
                    kX = kFewRows * kFewBlocks / 4 / kFewThreads;
      const int end = min(kFewCols, (int)(a.N - n0)) * kblocks + ws_rem;
      const int per = kblocks / 4, total = kFewRows * per;
      u32x4 t[kW];
      uint32_t q[kX], r[RES ? kX : 1];
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const int at = 16 * (tid + kFewThreads * i);
        t[i] = __builtin_amdgcn_raw_buffer_load_b128(rws, at < end ? (uint32_t)at : kNowhere, 0, 0);
      }
      load_w(b0, s0);
      __builtin_amdgcn_sched_barrier(0);   // (Before the row indices are waited for.)
      load_x(b0, s0);
#pragma unroll
      for (int i = 0; i < kX; ++i) {
        const int n = tid + kFewThreads * i, at = min(n / per, kFewRows - 1);
        const uint32_t o = x_start(at);
        const uint32_t from = n < total && o != kNowhere ? o + 4 * (n - at * per) : kNowhere;
        q[i] = __builtin_amdgcn_raw_buffer_load_b32(rqs, from, 0, 0);
        if constexpr (RES) r[i] = __builtin_amdgcn_raw_buffer_load_b32(rrs, from, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kW; ++i) {
        const int at = 16 * (tid + kFewThreads * i);
        if (at < end) *reinterpret_cast<u32x4 *>(lds + at) = t[i];
      }
#pragma unroll
      for (int i = 0; i < kX; ++i) {
        const int n = tid + kFewThreads * i;       // (Rows are dense: stride is kblocks.)
        if (n < total) {
          *reinterpret_cast<uint32_t *>(ql + 4 * n) = q[i];
          if constexpr (RES) *reinterpret_cast<uint32_t *>(rl + 4 * n) = r[i];
        }
      }
    } else {
      const int nb = min(kblocks - cb, kFewBlocks);
      load_w(b0, s0);
      load_x(b0, s0);
      stage(rws, wl, kFewCols, cb, nb, [&](int at) {
        return n0 + at < a.N ? (uint32_t)(ws_rem + at * kblocks) : kNowhere;
      });
      stage(rqs, ql, kFewRows, cb, nb, x_start);
      if constexpr (RES) stage(rrs, rl, kFewRows, cb, nb, x_start);
    }
    __syncthreads();
    for (int s = s0;;) {
      multiply(b0, s);
      s += U;
      if (s >= s1) break;
      load_w(b0, s);
      load_x(b0, s);
    }
  }
  __syncthreads();
  v4f(*partial)[kFrags][64] = reinterpret_cast<v4f(*)[kFrags][64]>(lds);
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
template <bool RES, bool ZBF16, bool GK, bool FAST>
__global__ __launch_bounds__(Mid::kThreads, 3) void rfq_gemm_experts_both_kernel(
    ExpertsGemm a, ExpertTiles many, ExpertTiles few, int tiles) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  if ((int)blockIdx.x < tiles)
    many_tile<Mid, Mid, RES, ZBF16, GK>(a, many);
  else
    few_tile<RES, ZBF16, FAST>(a, few, (int)blockIdx.x - tiles, smem);
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

// Slots up to which an expert runs a few-row tile: all that one holds (60 experts of 2048 x
// 1408, 512 tokens of 4 choices: 37.5 us up to 8, 32.9 up to 16; 8 experts of 4096 x 4096, 16
// tokens of 2: 21.6 and 15.0, but 64 tokens 23.5 and 26.2).
constexpr int kFewSlots = kFewRows;

template <bool RES, bool ZBF16, bool GK, bool FAST>
hipError_t launch_both(const ExpertsGemm &g, const ExpertTiles &ex, hipStream_t stream) {
  constexpr int kMid = lds_bytes<Mid, RES, ZBF16>(), kFew = few_lds_bytes(kFewK);
  constexpr int kMost = kMid > kFew ? kMid : kFew;
  auto kern = rfq_gemm_experts_both_kernel<RES, ZBF16, GK, FAST>;
  static std::atomic<bool> attr_done[kMaxDevices];
  const hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), kMost);
  if (e != hipSuccess) return e;
  ExpertTiles many = ex, few = ex;
  many.above = few.most = kFewSlots;
  // At most P / (kFewSlots + 1) experts have more than kFewSlots slots; an expert with fewer has
  // one tile.
  const int64_t experts = std::min<int64_t>(g.E, g.P / (kFewSlots + 1));
  const int64_t tiles = experts ? many_tiles<Mid>(g.P, experts, g.N) : 0;
  const int64_t rest = few_tiles(std::min<int64_t>(g.P, g.E), g.N);
  const int bytes = experts ? kMost : few_lds_bytes(g.K);
  kern<<<(unsigned)(tiles + rest), Mid::kThreads, bytes, stream>>>(g, many, few, (int)tiles);
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

// 256 x 256 tiles from 96 slots an expert where 128 x 128 ones would number two a CU (8 experts
// of 4096 x 4096: 256 slots each 51.6 us, both 62; 128 each, 384 tiles, 46 and 38).
//
// P counts the pairs that a share of a layer drops as well, so that a share's experts have fewer
// slots than the rule takes them to have.  8 choices, K = 2048, us with these tiles and with
// both: 64 of 128 experts of 1536 rows, 1024 tokens 49.4 and 45.7, 4096 tokens 88 and 96; 16 of 128
// experts of 4096 rows, 256 tokens 17.1 and 18.0, 1024 tokens 33.5 and 26.2, 4096 tokens 63 and 66;
// of 1536 rows, 1024 tokens 25.1 and 16.2, 4096 tokens 28.7 and 27.5.
bool use_many(const ExpertsGemm &g) {
  return g.P >= 96 * (int64_t)g.E && (g.P / 128 + g.E / 2) * ((g.N + 127) / 128) >= 512;
}
}  // namespace

// The tiles of any of the launches, in work items.
bool gemm_experts_fits(int64_t P, int64_t E, int64_t N) {
  return (P / 128 + 2 * E) == 0 || (N + 63) / 64 <= ((1 << 24) - 16) / (P / 128 + 2 * E);
}

hipError_t launch_gemm_experts(const ExpertsGemm &g, bool z_bf16, hipStream_t stream) {
  const ExpertTiles ex{g.offsets, g.rows, g.E, (int)g.P, 0, INT32_MAX};
  const bool gk = g.K % (kStageK * kGroup) != 0, fast = g.K % 128 == 0 && g.K <= kFewK;
  auto go = [&](auto res, auto zb) {
    constexpr bool R = decltype(res)::value, Z = decltype(zb)::value;
    if (use_many(g))
      return gk ? launch_many<R, Z, true>(g, ex, stream) : launch_many<R, Z, false>(g, ex, stream);
    if (fast)
      return gk ? launch_both<R, Z, true, true>(g, ex, stream)
                : launch_both<R, Z, false, true>(g, ex, stream);
    return gk ? launch_both<R, Z, true, false>(g, ex, stream)
              : launch_both<R, Z, false, false>(g, ex, stream);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (g.rc) return z_bf16 ? go(Yes{}, Yes{}) : go(Yes{}, No{});
  return z_bf16 ? go(No{}, Yes{}) : go(No{}, No{});
}

}  // namespace rfq
