// Attention over the MXFP4 cache for requests with many rows (prompts): workgroups of
// 128 rows of one head.
//
// The arithmetic is attention.hip's (S^T = K Q^T, O^T = V^T P^T on the bf16 matrix
// cores, a running maximum and sum a row); here the matrix products are the work: 4 D
// operations for each row and token against 2 D code bytes / 32 rows a token and wave.
// Four waves of 32 rows share each tile of 64 tokens, which is decoded to bf16 once, by
// all of them, into LDS, so that decoding costs a quarter of what it does in a wave of
// its own.  32 x 32 x 16 products: a lane holds one row's scores of half a tile's
// tokens, the other half is in lane ^ 32, and P again goes from one product to the next
// in the lane's registers.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "attention_device.h"
#include "kv.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

__device__ __forceinline__ v16f mma32(const u32x4 &a, const u32x4 &b, const v16f &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int D>
struct Wide {
  static constexpr int kRows = 128, kTile = 64, kWaveRows = 32;
  static constexpr int kLanes = D / 32;                   // 32-channel blocks of a token
  static constexpr int kBlocks = kTile * kLanes;          // of a tile
  static constexpr int kLoads = (kBlocks + kThreads - 1) / kThreads;
  static constexpr int kPart = kTile * 2 * D;             // bytes of a tile's keys (values)
  static constexpr int kLds = 4 * kPart;                  // two tiles
  // Rows of 2 D bytes.  Keys in units of 16 bytes (an operand's 8 channels), values in
  // units of 32 (the 16 channels that a transposing read takes), exchanged by the
  // token so that the rows that are read at once lie in different banks.
  static __device__ __forceinline__ int key(int token, int unit) {
    return token * 2 * D + (unit ^ (D == 64 ? token >> 1 & 7 : token & 15)) * 16;
  }
  static __device__ __forceinline__ int value(int token, int unit) {
    return token * 2 * D + (unit ^ (D == 64 ? token >> 1 & 3 : token & 7)) * 32;
  }
};

// Requests with more than few_rows rows (the others are attention.hip's).  The row
// tiles of request b are numbered from floor(start_b group / 128) + b, which leaves
// room for every row.  Matrix and vector units run side by side: a wave's step k does
// the softmax of tile k, whose scores it has, the scores of tile k + 1 in the registers
// that each half of it leaves, and O += V P of tile k with the decoding of keys k + 2 and
// values k + 1 into the LDS buffers that step k - 1 left.  One barrier a step.
template <int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void kv_attention_wide_kernel(
    const AttentionArgs a, int few_rows, int tiles) {
  using S = Wide<D>;
  constexpr int LT = S::kLanes, KS = D / 16, CT = D / 32, L = S::kLoads;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // [2] keys, [2] values
  __shared__ int lds_have[4][S::kTile / 16];              // whether a piece has a block
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  // Neighbouring workgroups take different heads (where these number 8, a head's
  // blocks stay in one XCD's L2); the last row tiles, with the most tokens, come first.
  const int head = blockIdx.x % a.heads;
  const int index = tiles - 1 - (int)(blockIdx.x / a.heads);
  auto first_tile = [&](int b) {
    return (int)((int64_t)min(max(a.starts[b], 0), a.T) * a.group / S::kRows) + b;
  };
  int b = 0, past = a.B;
  while (past - b > 1) {
    const int mid = (b + past) >> 1;
    if (first_tile(mid) <= index) b = mid;
    else past = mid;
  }
  const Request req = request<S>(a, b);
  const int rows = req.nq * a.group, rt = index - first_tile(b);
  if (rows <= few_rows || rt < 0 || rt >= req.row_tiles) return;

  // The lane's row, its queries as the right operand, what it sees.  A negative scale
  // goes into the queries' signs, so that the largest score is the largest product.
  const int row0 = rt * S::kRows, r = row0 + wave * S::kWaveRows + col;
  const int i = r / a.group, qh = head * a.group + (r - i * a.group);
  const bool real = r < rows;
  u32x4 qf[KS];
  const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    qf[k] = u32x4{0, 0, 0, 0};
    if (real) {
      qf[k] = *reinterpret_cast<const u32x4 *>(a.q + (req.start + i) * a.q_ts + qh * a.q_hs +
                                               16 * k + 8 * h);
      qf[k] ^= flip;
    }
  }
  // (At scale 0 a masked -infinity has to stay one.)
  const float c = fabsf(a.scale_log2) < 0x1p-126f ? 0x1p-126f : fabsf(a.scale_log2);
  const int pos = req.len - req.nq + i;
  const int hi = a.causal ? min(pos, req.len - 1) : req.len - 1;
  const int lo = a.window ? pos - a.window + 1 : 0;
  // What the wave's rows see: all of them from all_lo to all_hi, none outside any_lo to
  // any_hi; the workgroup's tiles.
  auto position = [&](int row) { return req.len - req.nq + min(row, rows - 1) / a.group; };
  const int w0 = row0 + wave * S::kWaveRows;
  const int p0 = position(w0), p1 = position(w0 + S::kWaveRows - 1);
  const int all_hi = a.causal ? p0 : req.len - 1, any_hi = a.causal ? p1 : req.len - 1;
  const int all_lo = a.window ? p1 - a.window + 1 : 0, any_lo = a.window ? p0 - a.window + 1 : 0;
  const int g_hi = a.causal ? position(row0 + S::kRows - 1) : req.len - 1;
  const int g_lo = a.window ? max(position(row0) - a.window + 1, 0) : 0;
  const int tile0 = g_lo / S::kTile, end = g_hi < 0 ? 0 : g_hi / S::kTile + 1;

  const int32_t *table = a.tables + (int64_t)b * a.width;
  // The thread's blocks of a tile: number n = tid + 256 l, block n % LT of token n / LT.
  // Scale bytes of both come with the keys; the values follow a step later.
  u32x4 kc[L], vc[L];
  uint32_t ks[L], vs[L], vs_next[L];
  int64_t at[L];
  int id[L], ok[L];
  auto look_up = [&](int tile) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int t = tile * S::kTile + (tid + kThreads * l) / LT;
      id[l] = -1;
      if (tid + kThreads * l < S::kBlocks && t < req.len) id[l] = table[t >> a.page_shift];
    }
  };
  auto fetch_keys = [&](int tile) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int n = tid + kThreads * l, t = tile * S::kTile + n / LT;
      ok[l] = (uint32_t)id[l] < (uint32_t)a.blocks;
      const int64_t row =
          (((int64_t)(ok[l] ? id[l] : 0) * a.heads + head) << a.page_shift) + (t & (a.page - 1));
      at[l] = row * LT + n % LT;
      kc[l] = reinterpret_cast<const u32x4 *>(a.k_codes)[at[l]];
      ks[l] = a.k_scales[at[l]];
      vs_next[l] = a.v_scales[at[l]];
    }
  };
  auto fetch_values = [&] {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      vc[l] = reinterpret_cast<const u32x4 *>(a.v_codes)[at[l]];
      vs[l] = vs_next[l];
    }
  };
  // A block that is NaN (a value byte that bf16 does not hold) makes its token's scores
  // NaN; the values in LDS are finite, so that a masked P gives 0.
  auto decode_keys = [&](int tile) {
    uint8_t *keys = lds + (tile & 1) * S::kPart;
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int n = tid + kThreads * l, token = n / LT, block = n % LT;
      if (S::kBlocks % kThreads == 0 || n < S::kBlocks) {
        if (n % (16 * LT) == 0) lds_have[tile & 3][token / 16] = ok[l];
        const bool nan = ks[l] == 0xFFu || vs_next[l] >= 0xFDu;
        const float sk = scale_operand(ks[l]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          u32x4 x = decode_bf16(kc[l][w], sk);
          if (w == 0 && nan) x[0] = 0x7FC07FC0u;
          *reinterpret_cast<u32x4 *>(keys + S::key(token, 4 * block + w)) = x;
        }
      }
    }
  };
  auto decode_values = [&](int tile) {
    uint8_t *vals = lds + (2 + (tile & 1)) * S::kPart;
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int n = tid + kThreads * l, token = n / LT, block = n % LT;
      if (S::kBlocks % kThreads == 0 || n < S::kBlocks) {
        const float sv = scale_operand(vs[l] < 0xFDu ? vs[l] : 0u);
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<u32x4 *>(vals + S::value(token, 2 * block + w / 2) + 16 * (w % 2)) =
              decode_bf16(vc[l][w], sv);
      }
    }
  };

  v16f o[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) o[t] = v16f{};
  float m = neg_inf(), sum = 0.0f;                        // m: in units of log2
  // Whether some row of the wave sees something of a tile.
  auto seen = [&](int tile) {
    return tile < end && tile * S::kTile <= any_hi && (tile + 1) * S::kTile > any_lo;
  };
  v16f s[2];
  // Half t of a tile's scores.
  auto score = [&](int tile, int t) {
    const uint8_t *keys = lds + (tile & 1) * S::kPart;
    s[t] = v16f{};
#pragma unroll
    for (int k = 0; k < KS; ++k)
      s[t] = mma32(*reinterpret_cast<const u32x4 *>(keys + S::key(32 * t + col, 2 * k + h)), qf[k],
                   s[t]);
  };

  if (tile0 < end) {
    look_up(tile0);
    fetch_keys(tile0);
    fetch_values();
    look_up(tile0 + 1);
    decode_keys(tile0);
    fetch_keys(tile0 + 1);
    look_up(tile0 + 2);
    decode_values(tile0);
    fetch_values();
    decode_keys(tile0 + 1);
    fetch_keys(tile0 + 2);
    look_up(tile0 + 3);
    __syncthreads();
    score(tile0, 0);
    score(tile0, 1);
  }
  for (int tile = tile0; tile < end; ++tile) {
    const int t0 = tile * S::kTile;
    const bool now = seen(tile);
    if (now) {
      int have[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) have[p] = lds_have[tile & 3][p];
      const bool whole = (have[0] & have[1] & have[2] & have[3]) && t0 >= all_lo &&
                         t0 + S::kTile - 1 <= all_hi;
      if (!__builtin_amdgcn_readfirstlane(whole)) {
        asm volatile("");                                 // (a branch, not selects)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int tok = t0 + 32 * t + 8 * (e / 4) + 4 * h + e % 4;
            const bool see = tok >= lo && tok <= hi && have[2 * t + e / 8];
            s[t][e] = see ? s[t][e] : neg_inf();
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top),
                                                         __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * c;
      // The reference follows the maximum only where P would pass 2^8.
      if (__any(top > m + 8.0f)) {
        asm volatile("");
        const float up = fmaxf(top, m);
        const float f = exp2_hw(m - (up == neg_inf() ? 0.0f : up));
        sum *= f;
#pragma unroll
        for (int t = 0; t < CT; ++t) o[t] *= f;
        m = up;
      }
    }
    u32x2 pf[2][4];
    const float ref = m == neg_inf() ? 0.0f : m;
    auto weigh = [&](int t, int q) {
      float e[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        e[x] = exp2_hw(__builtin_fmaf(s[t][4 * q + x], c, -ref));
        sum += e[x];
      }
      const bf16x4 y = {(__bf16)e[0], (__bf16)e[1], (__bf16)e[2], (__bf16)e[3]};
      pf[t][q] = __builtin_bit_cast(u32x2, y);
    };
    if (now) {
#pragma unroll
      for (int q = 0; q < 4; ++q) weigh(0, q);
      score(tile + 1, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) weigh(1, q);
      score(tile + 1, 1);
      const uint8_t *vals = lds + (2 + (tile & 1)) * S::kPart;
      // Tokens 16 u + 4 h + 0..3 and + 8 of it: the order in which P holds them.
      const int l16 = lane & 15, half = lane >> 4 & 1;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const u32x4 p = {pf[u / 2][u % 2 * 2][0], pf[u / 2][u % 2 * 2][1],
                         pf[u / 2][u % 2 * 2 + 1][0], pf[u / 2][u % 2 * 2 + 1][1]};
        const int token = 16 * u + 4 * h + (l16 >> 2);
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          const u32x2 v0 = read_transposed(vals + S::value(token, 2 * t + half) + (l16 & 3) * 8);
          const u32x2 v1 =
              read_transposed(vals + S::value(token + 8, 2 * t + half) + (l16 & 3) * 8);
          o[t] = mma32(u32x4{v0[0], v0[1], v1[0], v1[1]}, p, o[t]);
        }
      }
    } else {
      score(tile + 1, 0);
      score(tile + 1, 1);
    }
    // (Tiles past the end are decoded and scored too: from places that exist, not used.)
    decode_values(tile + 1);
    fetch_values();
    decode_keys(tile + 2);
    fetch_keys(tile + 3);
    look_up(tile + 4);
    __syncthreads();
  }

  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum),
                                                     false, false);
  sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (!real) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *out = a.out + (req.start + i) * a.o_ts + qh * a.o_hs;
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bf16x4 y = {(__bf16)(o[t][4 * q] * inv), (__bf16)(o[t][4 * q + 1] * inv),
                        (__bf16)(o[t][4 * q + 2] * inv), (__bf16)(o[t][4 * q + 3] * inv)};
      *reinterpret_cast<u32x2 *>(out + 32 * t + 8 * q + 4 * h) = __builtin_bit_cast(u32x2, y);
    }
  if (a.lse && h == 0)
    a.lse[(int64_t)(req.start + i) * a.Hq + qh] =
        sum == 0.0f ? neg_inf() : (m + __builtin_amdgcn_logf(sum)) * kLn2;
}

std::atomic<bool> g_lds_limit[3][kMaxDevices];

template <int D>
hipError_t launch(const AttentionArgs &a, int few_rows, hipStream_t stream) {
  using S = Wide<D>;
  const hipError_t e = set_lds_limit(g_lds_limit[D == 64 ? 0 : (D == 128 ? 1 : 2)],
                                     (const void *)kv_attention_wide_kernel<D>, S::kLds);
  if (e != hipSuccess) return e;
  const int64_t tiles = (int64_t)a.T * a.group / S::kRows + a.B;
  kv_attention_wide_kernel<D><<<(unsigned)(tiles * a.heads), kThreads, S::kLds, stream>>>(
      a, few_rows, (int)tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_attention_wide(const AttentionArgs &a, int64_t D, int few_rows,
                                    hipStream_t stream) {
  if (D == 64) return launch<64>(a, few_rows, stream);
  if (D == 128) return launch<128>(a, few_rows, stream);
  return launch<256>(a, few_rows, stream);
}

}  // namespace rfq
