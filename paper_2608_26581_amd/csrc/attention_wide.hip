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
// in the lane's registers, rounded to the products' bf16 (2^-9 of each weight; the sum l
// adds the unrounded weights in fp32).  With what that rounding drops as a second operand
// the error against 64 bits is the bf16 result's own (0.0016, else 0.0023), but the products
// are half as many again: a prompt of 8192 tokens 807 us for 536 on the same card, two pieces
// of prompts 153 for 107.
//
// Measured, 32 heads over 8 cached heads of 128 channels: a prompt of 8192 tokens in 556
// us, 988 TFLOP/s of the 1225 that a large bf16 product reaches on the card.  The issue
// of instructions bounds it: the matrix units are busy 46% and the vector units 60% of
// the time, the exponentials and the maximum standing against each 32 products.  Eight waves of 32
// rows, 64 rows a wave and operands read 2 or 4 products ahead are not faster.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "attention_device.h"
#include "kv.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Products that an operand is read from LDS before it is used.
constexpr int kReadAhead = 3;

__device__ __forceinline__ v16f mma32(const u32x4 &a, const u32x4 &b, const v16f &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The two codes of byte w (a constant) to bf16 times their scale.
__device__ __forceinline__ uint32_t decode_pair(uint32_t c, float s, int w) {
  bf16x2 r;
  if (w == 0) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  else if (w == 1) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  else if (w == 2) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  return __builtin_bit_cast(uint32_t, r);
}

template <int D>
struct Wide {
  static constexpr int kWaves = 4, kThreads = 64 * kWaves;
  static constexpr int kWaveRows = 32, kRows = kWaves * kWaveRows, kTile = 64;
  static constexpr int kLanes = D / 32;                   // 32-channel blocks of a token
  static constexpr int kBlocks = kTile * kLanes;          // of a tile
  static constexpr int kLoads = (kBlocks + kThreads - 1) / kThreads;
  // With two threads for each block, one decodes the keys' and one the values'.
  static constexpr bool kRoles = kThreads >= 2 * kBlocks;
  // In LDS the keys are rows of channels, the values rows of tokens (transposed while
  // they are decoded: a transposing read takes twice the LDS time of a plain one), with
  // the channel of row r r % (D / 8) * 8 + r / (D / 8) and the tokens in the order in which P
  // holds them.  Rows are padded by 16 bytes so that what 16 lanes read or write at once
  // lies in different banks; all addresses are one of a few registers and a constant.
  static constexpr int kOctets = D / 8;
  static constexpr int kKeyPitch = 2 * D + 16, kValuePitch = 2 * kTile + 16;
  static constexpr int kKeys = kTile * kKeyPitch, kValues = D * kValuePitch;
  static constexpr int kScales = kBlocks;                 // the values' scale bytes [block][token]
  static constexpr int kLds = 2 * (kKeys + kValues + kScales);    // two tiles
};

// The request that row tile `index` is numbered for, and which of its tiles it is (there
// may be none).
template <class S>
__device__ __forceinline__ int request_of_tile(const AttentionArgs &a, int index, int &rt) {
  auto first = [&](int b) {
    return (int)((int64_t)min(max(a.starts[b], 0), a.T) * a.group / S::kRows) + b;
  };
  int b = 0, past = a.B;
  while (past - b > 1) {
    const int mid = (b + past) >> 1;
    if (first(mid) <= index) b = mid;
    else past = mid;
  }
  rt = index - first(b);
  return b;
}

// Requests with more than few_rows rows (the others are attention.hip's).  The row
// tiles of request b are numbered from floor(start_b group / 128) + b, which leaves
// room for every row.
//
// Matrix and vector units run side by side: in a step, half a tile of 32 tokens, a wave
// turns its scores S_j into P_j while the matrix cores compute S_(j+1) and add
// P_(j-1) V to O; the three are independent.  Their operands are read from LDS
// kReadAhead products ahead.  In a tile's second half the keys of the tile after the next and the
// values of the next are decoded into the buffers that the first half was the last to
// read, behind the tile's one barrier.
template <int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_attention_wide_kernel(
    const AttentionArgs a, int few_rows, int tiles, float *parts_o, float *parts_ml) {
  using S = Wide<D>;
  constexpr int LT = S::kLanes, KS = D / 16, CT = D / 32, L = S::kLoads;
  constexpr int kThreads = S::kThreads;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // [2] keys, [2] values
  __shared__ alignas(16) int lds_have[4][S::kTile / 16];              // whether a piece has a block
  uint8_t *const lds_v = lds + 2 * S::kKeys, *const lds_s = lds_v + 2 * S::kValues;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  // Neighbouring workgroups take different heads (where these number 8, a head's
  // blocks stay in one XCD's L2); the last row tiles, with the most tokens, come first.
  const int head = blockIdx.x % a.heads;
  const int index = tiles - 1 - (int)(blockIdx.x / a.heads);
  int rt;
  const int b = request_of_tile<S>(a, index, rt);
  const Request req = request<S>(a, b);
  const int rows = req.nq * a.group;
  if (rows <= few_rows || rt < 0 || rt >= req.row_tiles) return;

  // The lane's rows, one of each 32; their queries as the right operand, and what they
  // see.  A negative scale goes into the queries' signs, so that the largest score is the
  // largest product.
  const int row0 = rt * S::kRows, w0 = row0 + wave * S::kWaveRows;
  u32x4 qf[KS];
  int lo, hi;
  const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
  {
    const int r = w0 + col, i = r / a.group, qh = head * a.group + (r - i * a.group);
    const int pos = req.len - req.nq + i;
    hi = a.causal ? min(pos, req.len - 1) : req.len - 1;
    lo = a.window ? pos - a.window + 1 : 0;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[k] = u32x4{0, 0, 0, 0};
      if (r < rows) {
        qf[k] = *reinterpret_cast<const u32x4 *>(a.q + (req.start + i) * a.q_ts +
                                                    qh * a.q_hs + 16 * k + 8 * h);
        qf[k] ^= flip;
      }
    }
  }
  // (At scale 0 a masked -infinity has to stay one, and no product, below 2^128, may show:
  // the least fp32 value.)
  const float c = a.scale_log2 == 0.0f ? 0x1p-149f : fabsf(a.scale_log2);
  // What all of the wave's rows see: all_lo to all_hi; the workgroup's tiles.
  auto position = [&](int row) { return req.len - req.nq + min(row, rows - 1) / a.group; };
  const int p0 = position(w0), p1 = position(w0 + S::kWaveRows - 1);
  const int all_hi = a.causal ? p0 : req.len - 1, all_lo = a.window ? p1 - a.window + 1 : 0;
  const int g_hi = a.causal ? position(row0 + S::kRows - 1) : req.len - 1;
  const int g_lo = a.window ? max(position(row0) - a.window + 1, 0) : 0;
  int tile0 = g_lo / S::kTile, end = g_hi < 0 ? 0 : g_hi / S::kTile + 1;
  const int parts = gridDim.y, part = blockIdx.y;
  if (parts > 1) {                                        // this workgroup's share of the tiles
    const int share = (max(end - tile0, 0) + parts - 1) / parts;
    tile0 += part * share;
    end = min(end, tile0 + share);
  }

  const int32_t *table = a.tables + (int64_t)b * a.width;
  // The thread's part of a tile.  Keys: block n % LT of token n / LT, n = tid + 256 l.
  // Values, a tile later: 8 channels n % kOctets of the 4 tokens n / kOctets, which are in
  // the same piece of 16 tokens as its keys.
  static_assert(S::kRoles || S::kBlocks % kThreads == 0, "every thread has the same work");
  const int first_n = S::kRoles ? tid % S::kBlocks : tid;
  const bool keys_mine = !S::kRoles || wave < S::kBlocks / 64;
  const bool values_mine = !S::kRoles || !keys_mine;
  u32x4 kc[L], vc[L];                                     // vc: a token's 8 codes each
  uint32_t ks[L], vs[L];
  const uint32_t *v_from[L];
  float sv[L][4];
  int id[L], ok[L];
  auto look_up = [&](int tile) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      // (By pieces, so that all of a piece find the same.)
      const int t = tile * S::kTile + (first_n + kThreads * l) / (16 * LT) * 16;
      id[l] = -1;
      if (t < req.len) id[l] = table[t >> a.page_shift];
    }
  };
  auto fetch_keys = [&](int tile) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int n = first_n + kThreads * l, token = n / LT, quad = n / S::kOctets * 4;
      ok[l] = (uint32_t)id[l] < (uint32_t)a.blocks;
      const int64_t row = (((int64_t)(ok[l] ? id[l] : 0) * a.heads + head) << a.page_shift) +
                          ((tile * S::kTile + (token & ~15)) & (a.page - 1));
      if (keys_mine) {
        const int64_t at = (row + (token & 15)) * LT + n % LT;
        kc[l] = reinterpret_cast<const u32x4 *>(a.k_codes)[at];
        ks[l] = a.k_scales[at];
        vs[l] = a.v_scales[at];
      }
      v_from[l] = reinterpret_cast<const uint32_t *>(a.v_codes) +
                  (row + (quad & 15)) * S::kOctets + n % S::kOctets;
    }
  };
  auto fetch_values = [&] {
    if (!values_mine) return;
#pragma unroll
    for (int l = 0; l < L; ++l)
#pragma unroll
      for (int i = 0; i < 4; ++i) vc[l][i] = v_from[l][i * S::kOctets];
  };
  // Part w of the thread's keys and values to LDS.  A block that is NaN (a value byte
  // that bf16 does not hold) makes its token's scores NaN; the values in LDS are finite,
  // so that a masked P gives 0.
  auto decode_key = [&](int buf, int tile, int l, int w) {
    if (!keys_mine) return;
    const int n = first_n + kThreads * l, token = n / LT, block = n % LT;
    u32x4 x = decode_bf16(kc[l][w], scale_operand(ks[l]));
    if (w == 0) {
      if (ks[l] == 0xFFu || vs[l] >= 0xFDu) x[0] = 0x7FC07FC0u;
      lds_have[tile & 3][token / 16] = ok[l];             // (the same from all of a piece)
      lds_s[buf * S::kScales + block * S::kTile + token] = vs[l] < 0xFDu ? (uint8_t)vs[l] : 0;
    }
    *reinterpret_cast<u32x4 *>(lds + buf * S::kKeys + token * S::kKeyPitch + 64 * block + 16 * w) =
        x;
  };
  auto decode_value = [&](int buf, int l, int w) {
    if (!values_mine) return;
    const int n = first_n + kThreads * l, octet = n % S::kOctets, quad = n / S::kOctets;
    if (w == 0) {
      const uint32_t scales = *reinterpret_cast<const uint32_t *>(
          lds_s + buf * S::kScales + octet / 4 * S::kTile + 4 * quad);
#pragma unroll
      for (int i = 0; i < 4; ++i) sv[l][i] = scale_operand(c_byte(scales, i));
    }
    uint32_t x[4];                                        // channels 2 w and 2 w + 1 of a token
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = decode_pair(vc[l][i], sv[l][i], w);
    // Four tokens of a channel; quads of 16 tokens in the order 0, 2, 1, 3.
    uint8_t *to = lds_v + buf * S::kValues + (2 * w * S::kOctets + octet) * S::kValuePitch +
                  (quad >> 2) * 32 + (quad & 1) * 16 + (quad >> 1 & 1) * 8;
    *reinterpret_cast<u32x2 *>(to) = u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u),
                                           __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)};
    *reinterpret_cast<u32x2 *>(to + S::kOctets * S::kValuePitch) =
        u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u),
              __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
  };
  auto decode_keys = [&](int buf, int tile) {
#pragma unroll
    for (int x = 0; x < 4 * L; ++x) decode_key(buf, tile, x / 4, x % 4);
  };
  auto decode_values = [&](int buf) {
#pragma unroll
    for (int x = 0; x < 4 * L; ++x) decode_value(buf, x / 4, x % 4);
  };

  v16f o[CT], s[2];
  u32x2 pf[2][4];                                         // P of a half, 4 tokens each
  float m = neg_inf(), sum = 0.0f;                        // m: in units of log2
#pragma unroll
  for (int t = 0; t < CT; ++t) o[t] = v16f{};
#pragma unroll
  for (int q = 0; q < 4; ++q) pf[1][q] = u32x2{0, 0};
  // Operand k of a half's keys; operand (u, t) of its values (16 tokens u, 32 rows t).
  auto key_frag = [&](int buf, int t, int k) {
    return *reinterpret_cast<const u32x4 *>(lds + buf * S::kKeys + col * S::kKeyPitch + 16 * h +
                                            32 * t * S::kKeyPitch + 32 * k);
  };
  auto value_frag = [&](int buf, int t, int f) {
    return *reinterpret_cast<const u32x4 *>(lds_v + buf * S::kValues + col * S::kValuePitch +
                                            16 * h + f % CT * 32 * S::kValuePitch +
                                            (2 * t + f / CT) * 32);
  };
  auto weights = [&](const u32x2 (&p)[4], int f) {
    const int u = f / CT;
    return u32x4{p[2 * u][0], p[2 * u][1], p[2 * u + 1][0], p[2 * u + 1][1]};
  };

  if (tile0 < end) {
    look_up(tile0);
    fetch_keys(tile0);
    fetch_values();
    look_up(tile0 + 1);
    decode_keys(0, tile0);
    fetch_keys(tile0 + 1);
    look_up(tile0 + 2);
    __syncthreads();                                      // (the values' scales)
    decode_values(0);
    for (int i = tid * 16; i < S::kValues; i += kThreads * 16)       // (read with P = 0)
      *reinterpret_cast<u32x4 *>(lds_v + S::kValues + i) = u32x4{0, 0, 0, 0};
    fetch_values();
    decode_keys(1, tile0 + 1);
    fetch_keys(tile0 + 2);
    look_up(tile0 + 3);
    __syncthreads();
    s[0] = v16f{};
#pragma unroll
    for (int k = 0; k < KS; ++k) s[0] = mma32(key_frag(0, 0, k), qf[k], s[0]);
  }
  // Which pieces of a tile have a block: read a step before it is needed.
  auto find = [&](int tile) { return *reinterpret_cast<const i32x4 *>(lds_have[tile & 3]); };
  i32x4 have = {0, 0, 0, 0};
  if (tile0 < end) have = find(tile0);
  // Half T of a tile.
  auto step = [&](int tile, auto half) {
    constexpr int T = decltype(half)::value, N = 1 - T;
    const int buf = (tile - tile0) & 1;
    const int keys = buf ^ T;                             // of S_(j+1), half N
    const int vals = buf ^ N;                             // of P_(j-1), half N
    const int t0 = tile * S::kTile + 32 * T;
    constexpr int kAhead = kReadAhead < KS ? kReadAhead : KS;
    u32x4 kf[KS], vf[KS];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      kf[k] = key_frag(keys, N, k);
      vf[k] = value_frag(vals, N, k);
    }
    const int have0 = have[2 * T], have1 = have[2 * T + 1];
    const bool whole = (have0 & have1) && t0 >= all_lo && t0 + 31 <= all_hi;
    if (!__builtin_amdgcn_readfirstlane(whole)) {
      asm volatile("");                                   // (a branch, not selects)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int tok = t0 + 8 * (e / 4) + 4 * h + e % 4;
        const bool see = tok >= lo && tok <= hi && (e < 8 ? have0 : have1);
        s[T][e] = see ? s[T][e] : neg_inf();
      }
    }
    float x = s[T][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) x = fmaxf(x, s[T][e]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                       false, false);
    const float top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * c;
    const bool grows = top > m + 8.0f;
    // The reference follows the maximum only where P would pass 2^8, to a whole power
    // of two: P_(j-1), still to be multiplied, is scaled exactly.
    if (__any(grows)) {
      asm volatile("");
      const float up = fmaxf(ceilf(top), m);
      const float f = exp2_hw(m - (up == neg_inf() ? 0.0f : up));
      sum *= f;
#pragma unroll
      for (int t = 0; t < CT; ++t) o[t] *= f;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t p = pf[N][q][x];
          const bf16x2 y = {(__bf16)(__uint_as_float(p << 16) * f),
                            (__bf16)(__uint_as_float(p & 0xFFFF0000u) * f)};
          pf[N][q][x] = __builtin_bit_cast(uint32_t, y);
        }
      m = up;
    }
    float e[16];
    const float ref = m == neg_inf() ? 0.0f : m;
    s[N] = v16f{};
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (k + kAhead < KS) {
        kf[k + kAhead] = key_frag(keys, N, k + kAhead);
        vf[k + kAhead] = value_frag(vals, N, k + kAhead);
      }
      s[N] = mma32(kf[k], qf[k], s[N]);
      o[k % CT] = mma32(vf[k], weights(pf[N], k), o[k % CT]);
#pragma unroll
      for (int x = k * 16 / KS; x < (k + 1) * 16 / KS; ++x) {
        e[x] = exp2_hw(__builtin_fmaf(s[T][x], c, -ref));
        if (x % 4 == 3) {
          const bf16x4 y = {(__bf16)e[x - 3], (__bf16)e[x - 2], (__bf16)e[x - 1],
                            (__bf16)e[x]};
          u32x2 &p = pf[T][x / 4];
          p = __builtin_bit_cast(u32x2, y);
          sum += (e[x - 3] + e[x - 2]) + (e[x - 1] + e[x]);
          // (Not to be moved behind the products.)
          asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(sum));
        }
      }
      if constexpr (T == 1) {
        if (k == 0) have = find(tile + 1);
        // The next codes to LDS, keys first; then the loads that take their registers.
#pragma unroll
        for (int x = k * 8 * L / KS; x < (k + 1) * 8 * L / KS; ++x) {
          if constexpr (S::kRoles) {
            if (x % 2 == 0) {
              decode_key(buf, tile + 2, x / 8, x / 2 % 4);
              decode_value(buf ^ 1, x / 8, x / 2 % 4);
            }
          } else {
            if (x < 4 * L) decode_key(buf, tile + 2, x / 4, x % 4);
            else decode_value(buf ^ 1, x / 4 - L, x % 4);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (T == 1) {
      fetch_values();
      fetch_keys(tile + 3);
      look_up(tile + 4);
    }
  };
  // (Tiles past the end are decoded and scored too: from places that exist, not used.)
  for (int tile = tile0; tile < end; ++tile) {
    step(tile, std::integral_constant<int, 0>{});
    __syncthreads();
    step(tile, std::integral_constant<int, 1>{});
  }
  if (tile0 < end) {
    const int buf = (end - 1 - tile0) & 1;
#pragma unroll
    for (int f = 0; f < KS; ++f)
      o[f % CT] = mma32(value_frag(buf, 1, f), weights(pf[1], f), o[f % CT]);
  }

  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum),
                                                     __float_as_uint(sum), false, false);
  const float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  const int r = w0 + col, i = r / a.group, qh = head * a.group + (r - i * a.group);
  if (r >= rows) return;
  if (parts > 1) {
    const int64_t at = ((int64_t)(index * a.heads + head) * parts + part) * S::kRows + r - row0;
    if (h == 0) {
      parts_ml[2 * at] = m;
      parts_ml[2 * at + 1] = l;
    }
    // Elements in the registers' order (the join's threads each take one position).
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const v16f &x = o[t];
        *reinterpret_cast<v4f *>(parts_o + at * D + 32 * t + 8 * q + 4 * h) =
            v4f{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
      }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t *out = a.out + (req.start + i) * a.o_ts + qh * a.o_hs;
  // Element e of tile t is row 32 t + 8 (e / 4) + 4 h + e % 4: 8 channels in the order of
  // memory are those whose rows are D / 8 apart.
#pragma unroll
  for (int g = 0; g < D / 16; ++g) {
    u32x4 y;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      float v[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // Row of the k-th channel of the lane's g-th octet (without 4 h).
        const int row = (k + x) * S::kOctets + g / 4 * 8 + g % 4;
        v[x] = o[row / 32][row % 32 / 8 * 4 + row % 4] * inv;
      }
      const bf16x2 p = {(__bf16)v[0], (__bf16)v[1]};
      y[k / 2] = __builtin_bit_cast(uint32_t, p);
    }
    *reinterpret_cast<u32x4 *>(out + 8 * (g / 4 * 8 + 4 * h + g % 4)) = y;
  }
  if (a.lse && h == 0)
    a.lse[(int64_t)(req.start + i) * a.Hq + qh] =
        l == 0.0f ? neg_inf() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The parts of the row tiles joined, in their order: thread = (row, 4 of the LDS rows that
// the channels have there).
template <int D>
__global__ __launch_bounds__(256) void kv_attention_wide_join_kernel(
    const AttentionArgs a, int few_rows, int tiles, int parts, const float *parts_o,
    const float *parts_ml) {
  using S = Wide<D>;
  constexpr int kLanes = D / 4, kRowsHere = 256 / kLanes;
  const int head = blockIdx.x % a.heads, index = blockIdx.x / a.heads;
  if (index >= tiles) return;
  int rt;
  const int b = request_of_tile<S>(a, index, rt);
  const Request req = request<S>(a, b);
  const int rows = req.nq * a.group;
  const int row = blockIdx.y * kRowsHere + threadIdx.x / kLanes, r = rt * S::kRows + row;
  if (rows <= few_rows || rt < 0 || rt >= req.row_tiles || r >= rows) return;
  const int c = threadIdx.x % kLanes * 4;
  const int64_t first = (int64_t)(index * a.heads + head) * parts * S::kRows + row;
  float top = neg_inf();
  for (int i = 0; i < parts; ++i) top = fmaxf(top, parts_ml[2 * (first + (int64_t)i * S::kRows)]);
  const float ref = top == neg_inf() ? 0.0f : top;
  float l = 0.0f;
  v4f x = {0, 0, 0, 0};
  for (int i = 0; i < parts; ++i) {
    const int64_t at = first + (int64_t)i * S::kRows;
    const float f = exp2_hw(parts_ml[2 * at] - ref);
    l += parts_ml[2 * at + 1] * f;
    x += *reinterpret_cast<const v4f *>(parts_o + at * D + c) * f;
  }
  x *= l == 0.0f ? 0.0f : 1.0f / l;
  const int i = r / a.group, qh = head * a.group + (r - i * a.group);
  uint16_t *out = a.out + (req.start + i) * a.o_ts + qh * a.o_hs;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int lds_row = c + e;
    const __bf16 y = (__bf16)x[e];
    out[lds_row % S::kOctets * 8 + lds_row / S::kOctets] = __builtin_bit_cast(uint16_t, y);
  }
  if (a.lse && c == 0)
    a.lse[(int64_t)(req.start + i) * a.Hq + qh] =
        l == 0.0f ? neg_inf() : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D>
hipError_t launch(const AttentionArgs &a, int few_rows, int parts, float *work,
                  hipStream_t stream) {
  using S = Wide<D>;
  static std::atomic<bool> limit[kMaxDevices];
  const auto kernel = kv_attention_wide_kernel<D>;
  hipError_t e = set_lds_limit(limit, (const void *)kernel, S::kLds);
  if (e != hipSuccess) return e;
  const int64_t tiles = wide_tiles(a.T, a.group, a.B), items = tiles * a.heads;
  float *ml = work ? work + items * parts * S::kRows * D : nullptr;
  kernel<<<dim3((unsigned)items, (unsigned)parts), S::kThreads, S::kLds, stream>>>(
      a, few_rows, (int)tiles, work, ml);
  if ((e = hipGetLastError()) != hipSuccess || parts == 1) return e;
  kv_attention_wide_join_kernel<D>
      <<<dim3((unsigned)items, (unsigned)(S::kRows * D / 4 / 256)), 256, 0, stream>>>(
          a, few_rows, (int)tiles, parts, work, ml);
  return hipGetLastError();
}

}  // namespace

int64_t wide_tiles(int64_t T, int64_t group, int64_t B) {
  return T * group / kWideRows + B;
}

int64_t wide_bytes(int64_t items, int parts, int64_t D) {
  return parts > 1 ? items * parts * kWideRows * (D + 2) * (int64_t)sizeof(float) : 0;
}

hipError_t launch_kv_attention_wide(const AttentionArgs &a, int64_t D, int few_rows, int parts,
                                    float *work, hipStream_t stream) {
  if (D == 64) return launch<64>(a, few_rows, parts, work, stream);
  if (D == 128) return launch<128>(a, few_rows, parts, work, stream);
  return launch<256>(a, few_rows, parts, work, stream);
}

}  // namespace rfq
