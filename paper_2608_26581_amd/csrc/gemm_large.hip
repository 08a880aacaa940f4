// RFQ product, large-tile kernel (Eq. 11, Algorithm 1 with phi = 1; phi = 0
// without the residual operand).
//
// Output tile 256 x 256 per workgroup of 8 waves (4 x 2, each wave 64 x 128
// = 2 x 4 fragments of 32 x 32), one workgroup per CU and two waves per SIMD:
// while one wave waits on LDS or global loads the other issues MFMAs.
// (Measured on 4096 x 4096 x 12288, bit-identical outputs: 4 waves of
// 128 x 128 with one wave per SIMD idled the matrix core on every wait; two
// 4-wave 128 x 256 workgroups per CU were 5-6% faster than that; this layout,
// which loads a quarter fewer operand bytes per output than the two
// workgroups, is another 4% faster.  The cost of the global loads lies in the
// load instructions themselves: pointing them at always-cached data does not
// change the time.)  Where the 256 x 256 tiles would leave CUs idle, the same
// code runs 128 x 128 tiles (4 waves of 64 x 64, up to three workgroups per
// CU) or 256 x 128 ones; each output is accumulated in the same order in all
// shapes, so they give the same bits.
//
// Instruction: v_mfma_scale_f32_32x32x64_f8f6f4 with E2M1 operands: lane l
// of an operand holds row (l mod 32) and 32 consecutive K values (one MX
// block) and supplies that block's scale byte; the 32 x 32 fp32 result gives
// lane l the rows 8a + 4(l/32) + 0..3 (a = 0..3) of column (l mod 32).  With
// weights as the first operand those are runs of four consecutive outputs
// of one row of Z.  (On gfx950 this form sustains about 7.6 PFLOP/s of FP4
// against about 6.1 for the 16x16x128 form in register-only loops.)
//
// One stage is 128 K values = 4 MX blocks = two k-steps: lane half h takes
// blocks 2h (k-step 0) and 2h+1 (k-step 1) - the contraction order inside an
// instruction is free as long as both operands use the same assignment - so
// a fragment is one 16-byte chunk per k-step and one 16-bit scale pair per
// stage (op_sel picks the byte).  Every weight fragment feeds the primary and
// the residual MFMA, which is the residual contraction sharing the weight
// tile.
//
// Pipeline per stage st (two LDS stage buffers of 52 KiB, one barrier per stage): the
// fragments of stage st are read from buffer st mod 2 and multiplied while
// stage st+1, held in registers, is written to the other buffer (its previous
// contents were last read before the barrier that ended stage st-1); then
// stage st+2 is fetched into the registers (with two stages in registers,
// for grids too small to cover the loads' latency, stage st+3).  Loads go through buffer
// descriptors (scalar base and size, a 32-bit offset per load).  Scale bytes
// arrive 16 per row every four stages (a 4-byte fetch per row and stage costs
// a whole L2 request for 4 useful bytes).  Inside LDS the 16-byte chunks of a
// row are XOR-swizzled by row, so the 16 rows served together by one 16-byte
// read hit distinct banks.
//
// Epilogue: each wave stages its results through LDS (padded rows) and
// writes Z with 16-byte stores covering whole row segments.  The SwiGLU
// epilogue instead takes the product of interleaved gate/up weights (32-row
// groups: gate rows 32g.., then up rows 32g..), so that columns 64g..64g+31
// of Z are g and 64g+32..64g+63 are u for the same 32 hidden units: it rounds
// both to bf16 as a bf16 Z would be, forms h = bf16(silu(g) u) and quantizes
// each 32-wide block of h (primary and residual, Eq. 8-10) from registers,
// with the same arithmetic as the standalone SwiGLU quantizer.
//
// Rows past M or N are clamped to the last row for loading (their results
// are never stored), so no load leaves its tensor.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "gemm_tile.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

#define RFQ_TILE_ARGS                                                                      \
  const uint8_t *__restrict__ qc, const uint8_t *__restrict__ qs,                          \
      const uint8_t *__restrict__ rc, const uint8_t *__restrict__ rs,                      \
      const uint8_t *__restrict__ wc, const uint8_t *__restrict__ ws, int64_t M, int64_t N, \
      int64_t K, void *__restrict__ z, SwigluOut so, const uint8_t *__restrict__ phi,      \
      int64_t ksplit

template <bool RES, bool ZBF16, bool SWIGLU, bool HRES, bool PHI, bool GK>
__global__ __launch_bounds__(Big::kThreads, 2) void rfq_gemm_large_kernel(RFQ_TILE_ARGS) {
  gemm_tile<Big, RES, ZBF16, SWIGLU, HRES, PHI, false, GK>(qc, qs, rc, rs, wc, ws, M, N, K, z, so,
                                                           phi, ksplit);
}

template <class C, bool RES, bool ZBF16, bool SWIGLU, bool HRES, bool PHI, bool GK>
__global__ __launch_bounds__(C::kThreads, C::kDepth > 1 ? 2 : 3) void rfq_gemm_mid_kernel(
    RFQ_TILE_ARGS) {
  gemm_tile<C, RES, ZBF16, SWIGLU, HRES, PHI, false, GK>(qc, qs, rc, rs, wc, ws, M, N, K, z, so,
                                                           phi, ksplit);
}

// K split over several workgroups per 128 x 128 tile: fp32 partial products.
template <class C, bool RES, bool GK>
__global__ __launch_bounds__(C::kThreads, C::kDepth > 1 ? 2 : 3) void rfq_gemm_split_kernel(
    RFQ_TILE_ARGS) {
  gemm_tile<C, RES, false, false, false, false, true, GK>(qc, qs, rc, rs, wc, ws, M, N, K, z, so,
                                                          phi, ksplit);
}
#undef RFQ_TILE_ARGS

// Z = sum of the S partial products p[s][M N], added in the order s = 0, 1,
// ...; four outputs per work item (V4: M N a multiple of 4), fp32 or bf16.
template <bool ZBF16, bool V4>
__global__ __launch_bounds__(256) void splitk_sum_kernel(const float *__restrict__ p, int S,
                                                         int64_t mn, void *__restrict__ z) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  if constexpr (V4) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < mn / 4; i += stride) {
      float4 a = reinterpret_cast<const float4 *>(p)[i];
      for (int s = 1; s < S; ++s) {
        const float4 b = reinterpret_cast<const float4 *>(p + s * mn)[i];
        a.x += b.x;
        a.y += b.y;
        a.z += b.z;
        a.w += b.w;
      }
      if constexpr (ZBF16)
        reinterpret_cast<uint2 *>(z)[i] = uint2{bf16x2_rne(a.x, a.y), bf16x2_rne(a.z, a.w)};
      else
        reinterpret_cast<float4 *>(z)[i] = a;
    }
  } else {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < mn; i += stride) {
      float a = p[i];
      for (int s = 1; s < S; ++s) a += p[s * mn + i];
      if constexpr (ZBF16)
        reinterpret_cast<uint16_t *>(z)[i] = (uint16_t)bf16_rne(a);
      else
        reinterpret_cast<float *>(z)[i] = a;
    }
  }
}

template <class C, bool RES, bool ZBF16, bool SWIGLU = false, bool HRES = false, bool PHI = false,
          bool GK = false>
hipError_t launch(const uint8_t *qc, const uint8_t *qs, const uint8_t *rc,
                  const uint8_t *rs, const uint8_t *wc, const uint8_t *ws,
                  int64_t M, int64_t N, int64_t K, void *z, hipStream_t stream,
                  const SwigluOut &so = SwigluOut{}, const uint8_t *phi = nullptr) {
  if constexpr (!SWIGLU && !GK)
    if (K % (kStageK * kGroup))
      return launch<C, RES, ZBF16, SWIGLU, HRES, PHI, true>(qc, qs, rc, rs, wc, ws, M, N, K, z,
                                                            stream, so, phi);
  using L = Layout<C, RES>;
  // The stage buffers or, where that is more, the waves' epilogue staging.
  constexpr int kEpiBytes = (C::kThreads / 64) * Epi<ZBF16>::kWaveBytes;
  constexpr int kBaseBytes = L::kBytes > kEpiBytes ? L::kBytes : kEpiBytes;
  void (*kern)(const uint8_t *, const uint8_t *, const uint8_t *, const uint8_t *,
               const uint8_t *, const uint8_t *, int64_t, int64_t, int64_t, void *, SwigluOut,
               const uint8_t *, int64_t);
  if constexpr (std::is_same<C, Big>::value)
    kern = rfq_gemm_large_kernel<RES, ZBF16, SWIGLU, HRES, PHI, GK>;
  else
    kern = rfq_gemm_mid_kernel<C, RES, ZBF16, SWIGLU, HRES, PHI, GK>;
  // LDS: the two stage buffers, then (PHI) the rows of the indicator map.
  constexpr int kMaxBytes = kBaseBytes + (PHI ? kPhiMapMaxBytes : 0);
  const int phi_bytes =
      PHI ? (int)(((C::kWaveRows * ((K + kPhiK - 1) / kPhiK)) + 15) / 16 * 16) : 0;
  static std::atomic<bool> attr_done[kMaxDevices];
  const hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), kMaxBytes);
  if (e != hipSuccess) return e;
  const int64_t ntiles = ((M + C::kBM - 1) / C::kBM) * ((N + C::kBN - 1) / C::kBN);
  kern<<<dim3((unsigned)ntiles), dim3(C::kThreads), kBaseBytes + phi_bytes, stream>>>(
      qc, qs, rc, rs, wc, ws, M, N, K, z, so, phi, K);
  return hipGetLastError();
}

int64_t mid_tiles(int64_t M, int64_t N) {
  return ((M + Mid::kBM - 1) / Mid::kBM) * ((N + Mid::kBN - 1) / Mid::kBN);
}

// K split into `parts` ranges of ksplit columns (a multiple of 512): the
// partial products go to work[parts][M][N] (fp32), then one pass adds them.
template <class C, bool RES, bool GK = false>
hipError_t launch_split(const uint8_t *qc, const uint8_t *qs, const uint8_t *rc,
                        const uint8_t *rs, const uint8_t *wc, const uint8_t *ws, int64_t M,
                        int64_t N, int64_t K, void *z, bool z_bf16, float *work, int parts,
                        int64_t ksplit, hipStream_t stream) {
  if constexpr (!GK)
    if (K % (kStageK * kGroup))
      return launch_split<C, RES, true>(qc, qs, rc, rs, wc, ws, M, N, K, z, z_bf16, work, parts,
                                        ksplit, stream);
  using L = Layout<C, RES>;
  auto kern = rfq_gemm_split_kernel<C, RES, GK>;
  static std::atomic<bool> attr_done[kMaxDevices];
  hipError_t e = set_lds_limit(attr_done, reinterpret_cast<const void *>(kern), L::kBytes);
  if (e != hipSuccess) return e;
  const int64_t ntiles = mid_tiles(M, N);
  kern<<<dim3((unsigned)(ntiles * parts)), dim3(C::kThreads), L::kBytes, stream>>>(
      qc, qs, rc, rs, wc, ws, M, N, K, work, SwigluOut{}, nullptr, ksplit);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  return launch_splitk_sum(work, parts, M * N, z, z_bf16, stream);
}

// Parts of K for the split product (1: no split), so that the parts x tiles
// workgroups fill the 256 CUs about once: 256 / tiles parts (at most 8) up to
// 128 tiles of 128 x 128, and for K >= 8192 512 / tiles (at most 4) up to
// 192 tiles; parts x tiles <= 512, so the partials take at most 32 MiB.
// Measured against the unsplit 128-wide tiles (random codes, bf16 Z): 64
// rows x 4096 x 12288 64.7 -> 18.5 us (8 parts); 129 rows 60.3 -> 23.9 (4);
// 256 rows 61.9 -> 28.5 (4); 512 rows 63.2 -> 44.3 (2); 64 rows x 5120 x
// 13824 80.9 -> 24.6 (6); 512 rows 72.5 -> 57.5 (3); 128 rows x 12288 x
// 4096 25.7 -> 22.1 (2).  With K = 4096 and 192 tiles (129 rows x 12288)
// two parts cost more than they save (21.3 -> 25.5 us).
int splitk_default_parts(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = mid_tiles(M, N);
  if (tiles <= 128) return (int)std::min<int64_t>(8, 256 / tiles);
  if (tiles <= 192 && K >= 8192) return (int)std::min<int64_t>(4, 512 / tiles);
  return 1;
}

// 128 x 128 tiles while they number fewer than two per CU of the 256 (up to
// three run on a CU at once).  Measured, same outputs either way: 0.53-0.58
// of the 256 x 256 time where those tiles fill at most a quarter of the CUs
// (129-256 rows x 12288 x 4096: 22-25 us against 40-43 us; 129-768 rows x
// 4096 x 12288: 60-67 us against 108-117 us), 0.8-0.96 at 384-480 tiles,
// 1.06-1.23 at 512-576.  Also where they are many and K is at most two stages,
// which is mostly prologue and epilogue, and those of a 256 x 256 tile nothing else
// on its CU overlaps (256 x 256 / 128 x 128: 4205 rows x 4204 x 256 plain 18.1 / 14.5,
// 2727 x 8724 x 256 plain 20.2 / 17.9, 2442 x 8447 x 192 plain 48.4 / 43.4; at 512 to
// 1023 tiles 0.94 to 1.08).
bool use_mid_tiles(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = mid_tiles(M, N);
  return tiles < 2 * 256 || (tiles >= 4 * 256 && K <= 2 * kStageK);
}

// Tall tiles where 128 x 128 ones number between one and two per CU and tall
// ones at most one.  Same bits.  Measured, 128 x 128 (Mid) against tall: 200
// rows x 24576 x 4096 (384 against 192 tiles) 35.6 -> 33.2 us, with the SwiGLU
// epilogue 38.9 -> 35.9, 512 rows x 12288 x 4096 37.2 -> 34.9 (plain 24.5 ->
// 21.7), 700 x 8192 x 4096 36.4 -> 34.2, 1000 x 5000 x 2912 (320 and 160) 29.8
// -> 29.6.  One stage in registers: 37.6 with the epilogue, the same without.
// At short K the start of the loop and the epilogue, which two workgroups on a
// CU overlap, take most of the time: from K = 1024 only (Mid against tall, 315 x
// 12544 x 512 plain 6.2 / 6.5 us, 370 x 15532 x 512 9.6 / 11.2; 828 x 5156 x 1024
// 13.0 / 13.0, 967 x 5888 x 1024 with a map 12.4 / 12.1), and with the SwiGLU
// epilogue, the longer one, from K = 2048 (432 rows x 13952 x 512 9.9 / 10.2,
// 1400 x 3264 x 1024 12.1 / 12.6, 6703 x 576 x 1536 14.6 / 15.6; 200 x 24576 x 4096
// above), plain 1536 (1047 x 5568 x 1024 8.3 / 8.8; 591 x 7360 x 1536 11.6 / 10.4).
constexpr int64_t kTallMinK = 1024, kTallSwigluMinK = 2048, kTallSwigluPlainMinK = 1536;
// Rows of Z that do not start at multiples of 16 bytes are stored in smaller
// pieces, the longest epilogue of the product: from K = 2048 (bf16 272 rows x 11019 x
// 1024 16.3 / 20.7, 4515 x 1365 x 1536 24.6 / 26.2, 302 x 10927 x 1536 plain 15.1 /
// 19.3, fp32 20.2 / 23.0; bf16 566 x 6860 x 2048 plain 16.7 / 13.9, 664 x 7924 x 2048
// 21.6 / 20.4, 888 x 6611 x 2048 29.7 / 30.2).  Not with one tile row, where the other
// shape has two: up to 192 rows from K = 512, whole rows of Z too (153 x 28884 x 2784
// 35.6 / 26.2, 165 x 18753 x 512 plain 15.4 / 11.0, 147 x 18176 x 512 7.5 / 7.0; 129 to 192
// rows at K = 512 to 1023 1.05 to 1.23 of its time, 193 to 256 0.95 to 1.02, below K =
// 512 0.92 to 1.27).
constexpr int64_t kTallBrokenRowsMinK = 2048, kTallOneRowMinK = 512, kTallOneRowMaxM = 192;
int64_t tall_min_k(int64_t M, int64_t N, bool z_bf16) {
  if (M <= kTallOneRowMaxM) return kTallOneRowMinK;
  return N % (z_bf16 ? 8 : 4) && M > Tall::kBM ? kTallBrokenRowsMinK : kTallMinK;
}
bool use_tall_tiles(int64_t M, int64_t N, int64_t K, int64_t min_k) {
  if (K < min_k) return false;
  const int64_t mid = mid_tiles(M, N);
  const int64_t tall = ((M + Tall::kBM - 1) / Tall::kBM) * ((N + Tall::kBN - 1) / Tall::kBN);
  return mid > 256 && mid < 2 * 256 && tall <= 256;
}

// MidDeep for `workgroups` 128 x 128 tiles (times parts of K): at most one
// per CU.  Same bits.  Measured, one stage against two in registers: 192
// tiles (129 and 256 rows x 12288 x 4096) 21.0 -> 18.3 and 23.5 -> 20.7 us,
// 64 and 128 tiles (200 and 512 rows x 4096 x 12288) 60.4 -> 48.5 and 63.1 ->
// 50.7, 256 tiles (1000 rows) 69.0 -> 64.4, split: 512 rows x 4096 x 12288
// 44.3 -> 41.8, 300 x 4096 x 11008 37.3 -> 32.3; at 320 tiles (1000 rows x
// 5000 x 2912), where three workgroups share a CU only without it, 29.7 ->
// 33.1, at 384 and 480 no gain.  Four stages gave no more than two.
// Not where a tile has so few stages that what is read ahead is most of K, and the
// registers' writes cost more than the wait (one / two; of the time, W not in L2, or
// us, W in L2): with the residual 0.93 to 0.97 below K = 512 at any number, 0.97 to 1.02
// at 512 (3 rows x 19904 x 512 with the SwiGLU epilogue 5.35 / 5.55 us), 0.98 to 0.99 up
// to 64 tiles at 1024 (3 x 64 x 1024 with that epilogue 6.5 / 6.75 us); without it 0.98
// to 1.00 up to 64 tiles to K = 512 (211 x 64 x 512 with it 4.0 / 4.2 us).  Beyond, 1.00
// to 1.08.
bool use_deep_tiles(int64_t workgroups, int64_t K, bool residual) {
  if (workgroups > 256) return false;
  if (!residual) return K > 512 || workgroups > 64;
  return K > 1024 || (K > 512 && workgroups > 64);
}

}  // namespace

hipError_t launch_splitk_sum(const float *work, int parts, int64_t mn, void *z, bool z_bf16,
                             hipStream_t stream) {
  const bool v4 = (mn % 4) == 0;
  const int64_t items = v4 ? mn / 4 : mn;
  const unsigned blocks = (unsigned)std::min<int64_t>((items + 255) / 256, 4096);
  if (z_bf16) {
    if (v4) splitk_sum_kernel<true, true><<<blocks, 256, 0, stream>>>(work, parts, mn, z);
    else splitk_sum_kernel<true, false><<<blocks, 256, 0, stream>>>(work, parts, mn, z);
  } else {
    if (v4) splitk_sum_kernel<false, true><<<blocks, 256, 0, stream>>>(work, parts, mn, z);
    else splitk_sum_kernel<false, false><<<blocks, 256, 0, stream>>>(work, parts, mn, z);
  }
  return hipGetLastError();
}

SplitPlan splitk_plan(int64_t M, int64_t N, int64_t K, int parts_wanted) {
  SplitPlan p{1, K, 0};
  const int64_t units = (K + kStageK * kGroup - 1) / (kStageK * kGroup);
  if (!use_mid_tiles(M, N, K) || units < 2) return p;
  int want = parts_wanted;
  if (want <= 0) want = splitk_default_parts(M, N, K);
  if (want < 2) return p;
  const int64_t per = (units + want - 1) / want;
  p.parts = (int)((units + per - 1) / per);
  if (p.parts < 2) return SplitPlan{1, K, 0};
  p.ksplit = per * kStageK * kGroup;
  p.work_bytes = (int64_t)p.parts * M * N * 4;
  return p;
}

hipError_t launch_gemm_large_split(const uint8_t *q_codes, const uint8_t *q_scales,
                                   const uint8_t *r_codes, const uint8_t *r_scales,
                                   const uint8_t *w_codes, const uint8_t *w_scales, int64_t M,
                                   int64_t N, int64_t K, void *z, bool z_bf16,
                                   const SplitPlan &plan, float *work, hipStream_t stream) {
  if (plan.parts < 2)
    return launch_gemm_large(q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, M, N, K,
                             z, z_bf16, stream);
  auto go = [&](auto tile) {
    using C = decltype(tile);
    if (r_codes)
      return launch_split<C, true>(q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, M, N,
                                   K, z, z_bf16, work, plan.parts, plan.ksplit, stream);
    return launch_split<C, false>(q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, M, N, K,
                                  z, z_bf16, work, plan.parts, plan.ksplit, stream);
  };
  return use_deep_tiles(mid_tiles(M, N) * plan.parts, plan.ksplit, r_codes != nullptr) ? go(MidDeep{}) : go(Mid{});
}

bool large_tiles_beat_few_rows(int64_t M, int64_t N, int64_t K) {
  if (M > 32 && N >= 16384 && K <= 2048 && K % 512) return true;
  return M > 64 && (N + Mid::kBN - 1) / Mid::kBN >= 96;
}

bool gemm_large_applies(const uint8_t *q_scales, const uint8_t *r_scales,
                        const uint8_t *w_scales, int64_t M, int64_t N, int64_t K) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(q_scales) |
                      reinterpret_cast<uintptr_t>(r_scales) |
                      reinterpret_cast<uintptr_t>(w_scales);
  // Byte offsets inside an operand are 32-bit; where K does not divide by 512
  // their top bit marks the loads past K.
  const int64_t limit = int64_t(1) << ((K % (kStageK * kGroup)) == 0 ? 32 : 31);
  return (a & 15) == 0 && M * (K / 2) < limit && N * (K / 2) < limit;
}

// 256-row tile rows that run 256 x 256 tiles where those do not fill their
// last round of 256 well: a last round of at most 64 tiles would run at a
// quarter of the chip for a whole tile time, so the tile rows of that round
// run 128 x 128 tiles in a second launch instead (1536 rows x 12288 x 4096:
// 101 -> 85 us; 4096 rows x 5120 x 13824: 330 -> 308 us).  Returns the
// number of tile rows of the 256 x 256 launch (all of them where nothing is
// peeled).
static int64_t big_tile_rows(int64_t M, int64_t N) {
  const int64_t ntm = (M + Big::kBM - 1) / Big::kBM, ntn = (N + Big::kBN - 1) / Big::kBN;
  const int64_t tiles = ntm * ntn, tail = tiles % 256;
  if (tail == 0 || tail > 64) return ntm;
  const int64_t rows = (tiles - tail) / ntn;
  return rows > 0 ? rows : ntm;
}

// Calls go(tile, first row, rows) for the tile shapes that M x N x K takes, with or
// without a map.
template <class Go>
static hipError_t on_tiles(int64_t M, int64_t N, int64_t K, bool residual, bool z_bf16, Go go) {
  auto mid = [&](int64_t row0, int64_t rows) {
    return use_deep_tiles(mid_tiles(rows, N), K, residual) ? go(MidDeep{}, row0, rows)
                                                           : go(Mid{}, row0, rows);
  };
  if (use_tall_tiles(M, N, K, tall_min_k(M, N, z_bf16))) return go(Tall{}, 0, M);
  if (use_mid_tiles(M, N, K)) return mid(0, M);
  const int64_t big_rows = std::min<int64_t>(big_tile_rows(M, N) * Big::kBM, M);
  const hipError_t e = go(Big{}, 0, big_rows);
  if (e != hipSuccess || big_rows == M) return e;
  // Both tile shapes accumulate every output in the same order, so the
  // peeled rows carry the bits the 256 x 256 tiles would give them.
  return mid(big_rows, M - big_rows);
}

hipError_t launch_gemm_large(const uint8_t *q_codes, const uint8_t *q_scales,
                             const uint8_t *r_codes, const uint8_t *r_scales,
                             const uint8_t *w_codes, const uint8_t *w_scales,
                             int64_t M, int64_t N, int64_t K, void *z, bool z_bf16,
                             hipStream_t stream) {
  return on_tiles(M, N, K, r_codes != nullptr, z_bf16, [&](auto tile, int64_t row0, int64_t rows) {
    using C = decltype(tile);
    // Activation rows [row0, row0 + rows) and the same rows of Z.
    const uint8_t *qc = q_codes + row0 * (K / 2), *qs = q_scales + row0 * (K / 32);
    const uint8_t *rc = r_codes ? r_codes + row0 * (K / 2) : nullptr;
    const uint8_t *rs = r_codes ? r_scales + row0 * (K / 32) : nullptr;
    void *zr = static_cast<uint8_t *>(z) + row0 * N * (z_bf16 ? 2 : 4);
    if (r_codes) {
      if (z_bf16)
        return launch<C, true, true>(qc, qs, rc, rs, w_codes, w_scales, rows, N, K, zr, stream);
      return launch<C, true, false>(qc, qs, rc, rs, w_codes, w_scales, rows, N, K, zr, stream);
    }
    if (z_bf16)
      return launch<C, false, true>(qc, qs, rc, rs, w_codes, w_scales, rows, N, K, zr, stream);
    return launch<C, false, false>(qc, qs, rc, rs, w_codes, w_scales, rows, N, K, zr, stream);
  });
}

hipError_t launch_gemm_large_phi(const uint8_t *q_codes, const uint8_t *q_scales,
                                 const uint8_t *r_codes, const uint8_t *r_scales,
                                 const uint8_t *w_codes, const uint8_t *w_scales,
                                 const uint8_t *phi, int64_t M, int64_t N, int64_t K, void *z,
                                 bool z_bf16, hipStream_t stream) {
  return on_tiles(M, N, K, true, z_bf16, [&](auto tile, int64_t row0, int64_t rows) {
    using C = decltype(tile);
    // row0 is a multiple of 256: whole rows of the map.
    const int64_t co = row0 * (K / 2), so = row0 * (K / 32);
    const uint8_t *pr = phi + row0 / kPhiRows * ((K + kPhiK - 1) / kPhiK);
    void *zr = static_cast<uint8_t *>(z) + row0 * N * (z_bf16 ? 2 : 4);
    if (z_bf16)
      return launch<C, true, true, false, false, true>(q_codes + co, q_scales + so, r_codes + co,
                                                       r_scales + so, w_codes, w_scales, rows, N,
                                                       K, zr, stream, SwigluOut{}, pr);
    return launch<C, true, false, false, false, true>(q_codes + co, q_scales + so, r_codes + co,
                                                      r_scales + so, w_codes, w_scales, rows, N, K,
                                                      zr, stream, SwigluOut{}, pr);
  });
}

hipError_t launch_gemm_swiglu(const uint8_t *q_codes, const uint8_t *q_scales,
                              const uint8_t *r_codes, const uint8_t *r_scales,
                              const uint8_t *wgu_codes, const uint8_t *wgu_scales,
                              int64_t M, int64_t Nh, int64_t K, uint8_t *hq_codes,
                              uint8_t *hq_scales, uint8_t *hr_codes, uint8_t *hr_scales,
                              uint16_t *h_out, hipStream_t stream) {
  const SwigluOut so{hq_codes, hq_scales, hr_codes, hr_scales, h_out, Nh};
  const int64_t N = 2 * Nh;
  auto go = [&](auto tile) {
    using C = decltype(tile);
    if (r_codes) {
      if (hr_codes)
        return launch<C, true, true, true, true>(q_codes, q_scales, r_codes, r_scales, wgu_codes,
                                                 wgu_scales, M, N, K, nullptr, stream, so);
      return launch<C, true, true, true, false>(q_codes, q_scales, r_codes, r_scales, wgu_codes,
                                                wgu_scales, M, N, K, nullptr, stream, so);
    }
    if (hr_codes)
      return launch<C, false, true, true, true>(q_codes, q_scales, r_codes, r_scales, wgu_codes,
                                                wgu_scales, M, N, K, nullptr, stream, so);
    return launch<C, false, true, true, false>(q_codes, q_scales, r_codes, r_scales, wgu_codes,
                                               wgu_scales, M, N, K, nullptr, stream, so);
  };
  if (!use_mid_tiles(M, N, K)) return go(Big{});
  if (use_tall_tiles(M, N, K, r_codes ? kTallSwigluMinK : kTallSwigluPlainMinK)) return go(Tall{});
  return use_deep_tiles(mid_tiles(M, N), K, r_codes != nullptr) ? go(MidDeep{}) : go(Mid{});
}

}  // namespace rfq
