// Attention of a step's queries over an MXFP4 key/value cache (block tables).
//
// For a key/value head, the rows are its group's query heads times the request's
// queries (row r: query r / group, head r % group).  With the keys' tile as the left
// operand the scores come out transposed, S^T = K Q^T: a lane holds one row's
// scores of 16 tokens (4 of each 16-token piece), which is the layout in which
// O^T = V^T P^T takes P as its right operand, so P goes from one product to the
// next in the lane's own registers.  The running maximum m, sum l and accumulator O
// of a row follow each tile of 64 tokens: with m' = max(m, max S), O and l are scaled
// by exp(m - m') and exp(S - m') V is added; exponentials are base 2 with log2(e)
// folded into the scale.
//
// Codes are decoded to bf16 in registers (exact: two significant bits and a
// power-of-two scale) and multiplied by the bf16 matrix cores with fp32 sums; l adds the
// fp32 weights, and for its product P is rounded to bf16 (2^-9 of each weight).  What that
// rounding drops as a second bf16 operand costs 4 to 7% here, and registers that spill (64
// ragged requests 24.7 -> 25.8 us a pass, 4 of 131072 tokens 122.5 -> 131.2), and takes the
// error against 64 bits from 0.0016 to 0.0015, which is the bf16 result's own.
//
// The FP4 matrix instructions could take the keys' codes as they are against q split in
// two FP8 terms, but their sums keep about 2^-18 of the terms' sum (measured on
// 16 x 16 x 128; bf16: 2^-25), which shows in lse.
//
// What the rows share, the codes, is the traffic: D + D / 16 bytes a token and head for
// keys and values.  A wave reads them in the order of memory, 1 KB a load; the keys go
// through its LDS rows as codes, to where the operand takes them, the values as bf16, from
// which the transposing read takes them token by token.  The tokens of all requests and
// heads are one line of work cut into equal shares, one a workgroup, whatever the lengths
// are; items that a cut divides are joined by a second kernel.
//
// Measured, 8 cached heads of 128 channels: 4 requests of 131072 tokens, 40 heads of q, in
// 119.7 us and the join 6.6 (4.8 TB/s of the 5.1 that a large copy reaches on the card:
// bandwidth bounds it); with 32 of q 64 requests of 1 to 8192 tokens, 54670 in all, 20.4 + 4.8
// us (latency: a share is a few steps of a wave); one of 700 tokens, whole items, 9.8 us
// (latency: the lookups, three loads of codes one after another, and joining the waves).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "attention_device.h"
#include "kv.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

// Workgroups that the split kernel's work is divided over: three per CU where the
// registers allow three waves a SIMD, else two.  64 channels allow four, which long work
// takes (requests' heads times tokens): 4 requests of 131072 tokens and 8 heads 78.3 us, with
// three 85.5, but 64 requests of 2000 29.3 and 28.6.
constexpr int split_groups(int64_t D, int nt, int64_t heads, int64_t tokens) {
  if (nt == 2 || D == 256) return 512;
  return D == 64 && tokens >= (int64_t(1) << 21) / heads ? 1024 : 768;
}
// An item's queries, its first loads and the joining of the waves take about as long
// as this many tiles.
constexpr int kItemCost = 4;
// Workgroups of a launch, and the tokens of a part of the wide kernel's, at least.
constexpr int64_t kMaxGrid = int64_t(1) << 20;
constexpr int64_t kLeastPart = 256;

// ---- the shapes and the requests

// Tokens of a unit of work.
constexpr int kUnit = 64;

// D channels, NT 16-row fragments, P 16-token pieces a step of a wave: P = 4, or 2 where
// there is little work, whose steps more waves share: up to kLittle units a workgroup (8
// requests of 8000 tokens, 10.7 units: 25.9 us, with 4 28.2; 64 of 8000, 87 units: 129 and
// 122); and for 256 channels, whose codes would not fit the registers otherwise.
constexpr int kLittle = 16;
template <int D, int NT, int P>
struct Shape {
  static constexpr int kRows = 16 * NT, kPieces = P, kTile = 16 * P;   // kTile: of a step
  static constexpr int kWords = D / 32;                  // code dwords of a lane and token
  static constexpr int kLoads = kTile * D / 2 / 1024;    // 16-byte loads of a tile's codes
  static constexpr int kLanes = D / 32;                  // lanes of a token in a load
  static constexpr int kTokens = 64 / kLanes;            // tokens of a load
  static constexpr int kPitch = 2 * D + 32;              // bytes of a value row in LDS
  static constexpr int kCols = D / 16;                   // 16-channel tiles of O
  static constexpr int kWaveLds = 32 * kPitch;           // >= 16 * D * 4
};

// Units of work of an item (a head's row tile of a request): kUnit tokens each, and
// kItemCost for what an item costs besides; without a split one.
__device__ __forceinline__ int item_units(const Request &r, bool split) {
  return split ? r.tiles + kItemCost : 1;
}
__device__ __forceinline__ int64_t units(const AttentionArgs &a, const Request &r, bool split) {
  if (r.nq * a.group > a.most_rows) return 0;
  return (int64_t)a.heads * r.row_tiles * item_units(r, split);
}

// One part of a (request, head, row tile): where its partial result goes.
struct Partial {
  float *o;                               // [groups * 2][ROWS][D]
  float *ml;                              // [groups * 2][ROWS][2]
  struct Item {
    int start, row0, rows, head;          // the request's first row of q; of its rows row0 on
    int parts;                            // 0: no such item
    int unused[3];
  } *item;                                // [groups] item whose first part ends the range
};

// A lane's part of a tile.  Codes of 1 KB a load, 16 bytes a lane in the order of
// memory: load i holds token i kTokens + lane / kLanes, block lane % kLanes of it (32
// channels, one scale byte).  ks: the keys' scale bytes as the operand needs them.
template <class S>
struct Codes {
  u32x4 k[S::kLoads], v[S::kLoads];
  uint32_t vs[S::kLoads];
  uint32_t ks[S::kPieces];                // 256 channels: two bytes
};

// Waves a SIMD that the registers have to allow (as split_groups counts on).
constexpr int wave_bound(int D, int NT, int waves) {
  if (NT == 2 || D == 256 || waves == 8) return 2;
  return D == 64 ? 4 : 3;
}

template <int D, int NT, int kWaves>
__global__ __launch_bounds__(64 * kWaves, wave_bound(D, NT, kWaves)) void kv_attention_kernel(
    const AttentionArgs a, const Partial part, int split) {
  // Steps of 32 tokens, of 64, or what the work asks for.
  constexpr bool kShort = NT == 1, kLong = D < 256 && kWaves == 4;
  constexpr int kThreads = 64 * kWaves;
  using U = Shape<D, NT, 4>;              // (what is the same for both)
  static_assert(U::kTile == kUnit, "requests are counted in units");
  __shared__ alignas(16) uint8_t lds_v[kWaves][U::kWaveLds];
  __shared__ float lds_ml[kWaves][U::kRows][2];
  __shared__ int64_t scan[kWaves];
  __shared__ int64_t found_at;
  __shared__ int found_b;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int wg = blockIdx.x, groups = gridDim.x;

  // This workgroup's range [u0, u1) of the units of all requests, and the request b
  // that u0 is in, whose first unit is base.  A lane holds one request of the 64 from
  // `held` on.
  int64_t total = 0, u0, u1, share, base;
  int b, held = 0;
  Request mine;
  auto range = [&] {
    share = (total + groups - 1) / groups;
    if (split && share < kWaves / 2 + kItemCost) share = kWaves / 2 + kItemCost;
    u0 = share * wg;
    u1 = u0 + share < total ? u0 + share : total;
  };
  auto hold = [&](int from) {
    held = from;
    mine = from + lane < a.B ? request<U>(a, from + lane) : Request{};
  };
  auto scanned = [&](int64_t n) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(n, d);
      if (lane >= d) n += o;
    }
    return n;
  };
  if (a.B <= 64) {
    hold(0);
    const int64_t n = units(a, mine, split), incl = scanned(n);
    total = lane_value(incl, 63);
    range();
    const uint64_t at = __ballot(incl - n <= u0 && u0 < incl);
    b = at ? __builtin_ctzll(at) : 0;
    base = lane_value(incl - n, b);
  } else {
    const int per = (a.B + kThreads - 1) / kThreads;
    const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    int64_t n = 0;
    for (int i = b0; i < b1; ++i) n += units(a, request<U>(a, i), split);
    const int64_t incl = scanned(n);
    if (lane == 63) scan[wave] = incl;
    __syncthreads();
    int64_t before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += scan[w];
      total += scan[w];
    }
    total = lane_value(total, 0);
    before += incl - n;
    range();
    if (u0 < u1 && before <= u0 && u0 < before + n) {
      int i = b0;
      for (;; ++i) {
        const int64_t k = units(a, request<U>(a, i), split);
        if (u0 < before + k) break;
        before += k;
      }
      found_b = i;
      found_at = before;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(u0 < u1 ? found_b : 0);
    base = lane_value(found_at, 0);
    hold(b);
  }
  if (part.item && tid == 0) part.item[wg].parts = 0;
  if (u0 >= u1) return;
  auto pick = [&](int i) {                // request i, of those held
    if (i >= held + 64) hold(i);
    const int from = i - held;
    return request<U>(a, __builtin_amdgcn_readlane(mine.start, from),
                      __builtin_amdgcn_readlane(mine.nq, from),
                      __builtin_amdgcn_readlane(mine.len, from));
  };
  Request req = pick(b);

  auto work = [&](auto pieces) {
    constexpr int P = decltype(pieces)::value;
    using S = Shape<D, NT, P>;
    uint8_t *vbuf = lds_v[wave];
    constexpr int L = S::kLoads, LT = S::kLanes, W = S::kWords;
    // The 16-byte units of a token's codes in LDS, exchanged so that the 16 tokens of
    // a piece read theirs from different banks.
    auto swizzle = [](int token) { return (token / (16 / LT)) & (LT - 1); };

    for (int64_t u = u0; u < u1;) {
      int64_t n = units(a, req, split);
      while (u >= base + n) {               // next request that has work
        base += n;
        req = pick(++b);
        n = units(a, req, split);
      }
      const int nk = item_units(req, split);
      const int64_t local = u - base;
      const int item = local >> 32 ? (int)(local / nk) : (int)((uint32_t)local / (uint32_t)nk);
      const int k0 = (int)(local - (int64_t)item * nk);
      const int head = item / req.row_tiles, rt = item - head * req.row_tiles;
      const int64_t left = u1 - u;
      const int k1 = (int)(left < nk - k0 ? k0 + left : nk);
      u += k1 - k0;
      // The first kItemCost units of an item are no tiles.
      if (split && k1 <= kItemCost) continue;
      const bool first = !split || k0 <= kItemCost, complete = first && k1 == nk;
      constexpr int kSteps = kUnit / S::kTile;
      const int tile0 = kSteps * (req.tiles0 + (first ? 0 : k0 - kItemCost));
      const int tile1 = kSteps * (req.tiles0 + (split ? k1 - kItemCost : req.tiles));

      // The lane's rows: one of each 16-row tile.
      const int rows = req.nq * a.group, row0 = rt * S::kRows;
      int lo[NT], hi[NT];
      u32x4 qf[NT][W];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int r = row0 + 16 * t + col, i = r / a.group, h = r - i * a.group;
        const int p = req.len - req.nq + i;
        hi[t] = a.causal ? min(p, req.len - 1) : req.len - 1;
        lo[t] = a.window ? p - a.window + 1 : 0;
#pragma unroll
        for (int w = 0; w < W; ++w) qf[t][w] = u32x4{0, 0, 0, 0};
        if (r < rows) {
          const uint16_t *q = a.q + (req.start + i) * a.q_ts +
                              (head * a.group + h) * a.q_hs + g * (D / 4);
#pragma unroll
          for (int w = 0; w < W; ++w) qf[t][w] = *reinterpret_cast<const u32x4 *>(q + 8 * w);
        }
      }
      // Tokens that every row sees: from all_lo to all_hi; none beyond [any_lo, any_hi].
      const int last_row = min(row0 + S::kRows, rows) - 1;
      const int i0 = row0 / a.group, i1 = last_row / a.group;
      const int p0 = req.len - req.nq + i0, p1 = req.len - req.nq + i1;
      const int all_hi = a.causal ? p0 : req.len - 1, any_hi = a.causal ? p1 : req.len - 1;
      const int all_lo = a.window ? p1 - a.window + 1 : 0;
      const int any_lo = a.window ? p0 - a.window + 1 : 0;

      v4f o[NT][S::kCols];
      float m[NT], l[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        m[t] = neg_inf();
        l[t] = 0.0f;
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) o[t][c] = v4f{0, 0, 0, 0};
      }

      const int32_t *table = a.tables + (int64_t)b * a.width;
      // A tile's first rows in the cache, by its pieces, and which of them have a block.
      int64_t row[P];
      uint32_t have = 0;
      auto locate = [&](int tile) {
        have = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int t0 = tile * S::kTile + 16 * p;
          int id = -1;
          if (t0 < req.len) id = table[t0 >> a.page_shift];
          const bool ok = (uint32_t)id < (uint32_t)a.blocks;
          have |= (uint32_t)ok << p;
          row[p] = (((int64_t)(ok ? id : 0) * a.heads + head) << a.page_shift) +
                   (t0 & (a.page - 1));
        }
      };
      // Load i of a lane, in units of 16 code bytes, so of scale bytes.
      auto unit_at = [&](int i) -> int64_t {
        if constexpr (D == 64) return (lane < 32 ? row[2 * i] : row[2 * i + 1]) * LT + (lane & 31);
        else if constexpr (D == 128) return row[i] * LT + lane;
        else return row[i / 2] * LT + (i % 2) * 64 + lane;
      };
      Codes<S> c;
      auto fetch_keys = [&] {
#pragma unroll
        for (int i = 0; i < L; ++i) c.k[i] = reinterpret_cast<const u32x4 *>(a.k_codes)[unit_at(i)];
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const uint8_t *ks = a.k_scales + row[p] * LT + col * LT + g * (D / 4) / 32;
          if constexpr (D == 256) c.ks[p] = *reinterpret_cast<const uint16_t *>(ks);
          else c.ks[p] = *ks;
        }
      };
      auto fetch_values = [&] {
#pragma unroll
        for (int i = 0; i < L; ++i) {
          c.v[i] = reinterpret_cast<const u32x4 *>(a.v_codes)[unit_at(i)];
          c.vs[i] = a.v_scales[unit_at(i)];
        }
      };

      // The wave's tiles: every kWaves-th of the range that some row sees.
      int tile = tile0 + wave;
      while (tile < tile1 && (tile + 1) * S::kTile <= any_lo) tile += kWaves;
      const int end = min(tile1, (any_hi + S::kTile) / S::kTile);
      if (tile < end) {
        locate(tile);
        fetch_keys();
        fetch_values();
      }
      for (; tile < end; tile += kWaves) {
        // Keys to LDS in the order of memory; then the next tile's take their registers.
        // (The next values follow when this tile's have been decoded.)
#pragma unroll
        for (int i = 0; i < L; ++i) {
          const int token = i * S::kTokens + lane / LT, unit = lane % LT ^ swizzle(token & 15);
          *reinterpret_cast<u32x4 *>(vbuf + (token * LT + unit) * 16) = c.k[i];
        }
        uint32_t ks[P];
#pragma unroll
        for (int p = 0; p < P; ++p) ks[p] = c.ks[p];
        const int t0 = tile * S::kTile;
        const uint32_t held_now = have;
        const bool whole = have == (1u << P) - 1 && t0 >= all_lo && t0 + S::kTile - 1 <= all_hi &&
                           t0 + S::kTile <= req.len;
        const bool more = tile + kWaves < end;
        if (more) {
          locate(tile + kWaves);
          fetch_keys();
        }
        // Keys whose own scale is NaN, or whose values bf16 does not hold, make their
        // token's scores NaN (values: looked for only where one is in the tile).
        bool bad[P], odd = false;
#pragma unroll
        for (int i = 0; i < L; ++i)
          odd |= c.vs[i] >= 0xFDu && t0 + i * S::kTokens + lane / LT < req.len;
#pragma unroll
        for (int p = 0; p < P; ++p)
          bad[p] = c_byte(ks[p], 0) == 0xFFu || (D == 256 && c_byte(ks[p], 1) == 0xFFu);
        if (__any(odd)) {
#pragma unroll
          for (int i = 0; i < L; ++i) {
            // Lanes of token: kLanes neighbours of load i.
            uint64_t m = __ballot(c.vs[i] >= 0xFDu);
#pragma unroll
            for (int p = 0; p < P; ++p) {
              const int token = 16 * p + col - i * S::kTokens;
              if (token >= 0 && token < S::kTokens)
                bad[p] |= (m >> (token * LT) & ((1u << LT) - 1)) != 0;
            }
          }
        }
        wave_sync();
        // Scores.
        v4f s[NT][P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
          for (int t = 0; t < NT; ++t) s[t][p] = v4f{0, 0, 0, 0};
          uint32_t kc[W];
          const uint8_t *src = vbuf + (16 * p + col) * (D / 2);
          if constexpr (D == 64) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(
                src + ((g / 2) ^ swizzle(col)) * 16 + (g & 1) * 8);
            kc[0] = x[0];
            kc[1] = x[1];
          } else {
#pragma unroll
            for (int w = 0; w < W; w += 4) {
              const u32x4 x = *reinterpret_cast<const u32x4 *>(
                  src + ((g * (W / 4) + w / 4) ^ swizzle(col)) * 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) kc[w + e] = x[e];
            }
          }
#pragma unroll
          for (int w = 0; w < W; ++w) {
            u32x4 kf = decode_bf16(kc[w], scale_operand(c_byte(ks[p], w / 4)));
            if (w == 0 && bad[p]) kf[0] = 0x7FC07FC0u;
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][p] = mma(kf, qf[t][w], s[t][p]);
          }
        }
        wave_sync();
        // Softmax statistics.
        u32x2 pf[NT][P];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float top = neg_inf();
#pragma unroll
          for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = s[t][p][i] * a.scale_log2;
              if (!whole) {
                const int tok = t0 + 16 * p + 4 * g + i;
                const bool see = tok >= lo[t] && tok <= hi[t] && (held_now >> p & 1);
                x = see ? x : neg_inf();
              }
              s[t][p][i] = x;
              top = fmaxf(top, x);
            }
          }
          top = fmaxf(across_max(top), m[t]);
          const float ref = top == neg_inf() ? 0.0f : top;
          if (__any(top > m[t])) {
            const float f = exp2_hw(m[t] - ref);
            l[t] *= f;
#pragma unroll
            for (int c = 0; c < S::kCols; ++c) o[t][c] *= f;
          }
          m[t] = top;
          float sum = 0.0f;
#pragma unroll
          for (int p = 0; p < P; ++p) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              e[i] = exp2_hw(s[t][p][i] - ref);
              sum += e[i];
            }
            const bf16x4 r = {(__bf16)e[0], (__bf16)e[1], (__bf16)e[2], (__bf16)e[3]};
            pf[t][p] = __builtin_bit_cast(u32x2, r);
          }
          l[t] += sum;
        }
        // Values, 32 tokens at a time; always finite: a masked token's P is 0 and has to
        // give 0.
#pragma unroll
        for (int half = 0; half < P / 2; ++half) {
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            const int i = half * (D / 64) + q;
            uint8_t *row = vbuf + (q * S::kTokens + lane / LT) * S::kPitch + lane % LT * 64;
            const float sc = scale_operand(c.vs[i] < 0xFDu ? c.vs[i] : 0u);
#pragma unroll
            for (int w = 0; w < 4; ++w)
              *reinterpret_cast<u32x4 *>(row + 16 * w) = decode_bf16(c.v[i][w], sc);
          }
          if (half == P / 2 - 1 && more) fetch_values();
          wave_sync();
          const uint8_t *src = vbuf + (4 * g + (col >> 2)) * S::kPitch + (col & 3) * 8;
#pragma unroll
          for (int c = 0; c < S::kCols; ++c) {
            const u32x2 v0 = read_transposed(src + 32 * c);
            const u32x2 v1 = read_transposed(src + 16 * S::kPitch + 32 * c);
            const u32x4 vf = {v0[0], v0[1], v1[0], v1[1]};
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const u32x4 pp = {pf[t][2 * half][0], pf[t][2 * half][1], pf[t][2 * half + 1][0],
                                pf[t][2 * half + 1][1]};
              o[t][c] = mma(vf, pp, o[t][c]);
            }
          }
          wave_sync();
        }
      }

      // The waves' results joined, a 16-row tile at a time: each scales its O by
      // exp2(m - M) and leaves it in its LDS rows; every thread adds some of them.
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        l[t] = across_sum(l[t]);
        if (g == 0) {
          lds_ml[wave][16 * t + col][0] = m[t];
          lds_ml[wave][16 * t + col][1] = l[t];
        }
      }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float top = neg_inf();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_ml[w][16 * t + col][0]);
        const float ref = top == neg_inf() ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
          sum += lds_ml[w][16 * t + col][1] * exp2_hw(lds_ml[w][16 * t + col][0] - ref);
        const float f = exp2_hw(m[t] - ref);
#pragma unroll
        for (int c = 0; c < S::kCols; ++c)
          *reinterpret_cast<v4f *>(vbuf + (c * 64 + lane) * 16) = o[t][c] * f;
        __syncthreads();
        const int r = row0 + 16 * t + col;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int slot = 2 * wg + (first ? 1 : 0);
        const int i = r / a.group, h = head * a.group + (r - i * a.group);
#pragma unroll
        for (int c = wave; c < S::kCols; c += kWaves) {
          v4f x = *reinterpret_cast<const v4f *>(lds_v[0] + (c * 64 + lane) * 16);
#pragma unroll
          for (int w = 1; w < kWaves; ++w)
            x += *reinterpret_cast<const v4f *>(lds_v[w] + (c * 64 + lane) * 16);
          if (complete) {
            if (r < rows) {
              x *= inv;
              const bf16x4 y = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
              *reinterpret_cast<u32x2 *>(a.out + (req.start + i) * a.o_ts + h * a.o_hs + 16 * c +
                                         4 * g) = __builtin_bit_cast(u32x2, y);
            }
          } else {
            *reinterpret_cast<v4f *>(part.o + ((int64_t)slot * S::kRows + 16 * t + col) * D +
                                     16 * c + 4 * g) = x;
          }
        }
        if (wave == 0 && g == 0) {
          if (complete) {
            if (a.lse && r < rows)
              a.lse[(int64_t)(req.start + i) * a.Hq + h] =
                  sum == 0.0f ? neg_inf() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
          } else {
            float *ml = part.ml + ((int64_t)slot * S::kRows + 16 * t + col) * 2;
            ml[0] = top;
            ml[1] = sum;
          }
        }
        __syncthreads();
      }
      if (!complete && first && tid == 0) {
        // Its other parts are the first of the following workgroups' ranges.
        const int parts = 1 + (int)((nk - k1 + share - 1) / share);
        part.item[wg] = {req.start, row0, rows, head, parts, {}};
      }
    }
  };
  if constexpr (kShort && kLong) {
    if (total <= (int64_t)kLittle * groups) work(std::integral_constant<int, 2>{});
    else work(std::integral_constant<int, 4>{});
  } else {
    work(std::integral_constant<int, kLong ? 4 : 2>{});
  }
}

constexpr int kJoinThreads = 256;

// The parts of the items that the split kernel began but did not finish in one
// workgroup: part 0 in slot 2 w + 1, the following ones in slots 2 (w + i).  Added in
// that order.
template <int D, int NT>
__global__ __launch_bounds__(kJoinThreads) void kv_attention_join_kernel(const AttentionArgs a,
                                                                     const Partial part) {
  constexpr int kRows = 16 * NT, kLanes = D / 4;         // kLanes: threads of a row
  const int wg = blockIdx.x;
  const Partial::Item it = part.item[wg];
  const int n = it.parts;
  const int row = blockIdx.y * (kJoinThreads / kLanes) + threadIdx.x / kLanes, r = it.row0 + row;
  if (n == 0 || r >= it.rows) return;
  const int lr = threadIdx.x % kLanes, c = 4 * lr;
  auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * wg + 1 : 2 * (wg + i)) * kRows + row; };
  // A lane of the row takes the statistics of every kLanes-th part; the first parts'
  // sums are on their way meanwhile.
  constexpr int kBatch = 8;
  v4f y[kBatch];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int e = 0; e < kBatch; ++e)
      y[e] = *reinterpret_cast<const v4f *>(part.o + slot(min(i0 + e, n - 1)) * D + c);
  };
  float top = neg_inf();
  for (int i = lr; i < n; i += kLanes) top = fmaxf(top, part.ml[slot(i) * 2]);
  fetch(0);
#pragma unroll
  for (int d = 1; d < kLanes; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == neg_inf() ? 0.0f : top;
  float sum = 0.0f, f = 0.0f;
  v4f x = {0, 0, 0, 0};
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    if (i0 % kLanes == 0) {
      f = 0.0f;
      if (i0 + lr < n) {
        const float *ml = part.ml + slot(i0 + lr) * 2;
        f = exp2_hw(ml[0] - ref);
        sum += ml[1] * f;
      }
    }
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const float w = __shfl(f, (i0 + e) % kLanes, kLanes);
      if (i0 + e < n) x += y[e] * w;
    }
    if (i0 + kBatch < n) fetch(i0 + kBatch);
  }
#pragma unroll
  for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d);
  x *= sum == 0.0f ? 0.0f : 1.0f / sum;
  const int i = r / a.group, h = it.head * a.group + (r - i * a.group);
  const bf16x4 z = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  *reinterpret_cast<u32x2 *>(a.out + (it.start + i) * a.o_ts + h * a.o_hs + c) =
      __builtin_bit_cast(u32x2, z);
  if (a.lse && c == 0)
    a.lse[(int64_t)(it.start + i) * a.Hq + h] =
        sum == 0.0f ? neg_inf() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int64_t partial_bytes(int64_t D, int nt, int64_t groups) {
  return groups * (2 * 16 * nt * (D + 2) * 4 + (int64_t)sizeof(Partial::Item));
}

template <int D, int NT, int kWaves>
hipError_t launch(const AttentionArgs &a, unsigned groups, float *work, hipStream_t stream) {
  using S = Shape<D, NT, 4>;
  const bool split = groups > 0;
  Partial p = {};
  unsigned grid;
  if (split) {
    p.o = work;
    p.ml = work + (int64_t)groups * 2 * S::kRows * D;
    p.item = reinterpret_cast<Partial::Item *>(p.ml + (int64_t)groups * 2 * S::kRows * 2);
    grid = groups;
  } else {
    // At least as many workgroups as there are items, within a launch's limits.
    const int64_t items = (up((int64_t)a.T * a.group, S::kRows) + a.B) * a.heads;
    grid = (unsigned)(items < kMaxGrid ? items : kMaxGrid);
  }
  kv_attention_kernel<D, NT, kWaves><<<grid, 64 * kWaves, 0, stream>>>(a, p, split);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !split) return e;
  const dim3 join(groups, (unsigned)up(S::kRows, kJoinThreads / (D / 4)));
  kv_attention_join_kernel<D, NT><<<join, kJoinThreads, 0, stream>>>(a, p);
  return hipGetLastError();
}

// What a call launches.  Requests of up to kFewRows rows (queries times group) never take
// the wide kernel, unless every request must have more (their sum and the largest say so;
// then a wrong hint costs time only, since the wide kernel takes rows of any number): two
// pieces of prompts over 16000 tokens take 9 us less without the other kernel's launches.
// Of 128 channels, eight requests of 64 rows over 3000 tokens take 33.8 us here and 40.4 in the wide
// kernel, of 128 rows 48.6 and 49.1, of 256 rows and 60000 tokens 912 and 885.
constexpr int kFewRows = 64;
struct Plan {
  bool few, wide;
  int few_rows;                           // the wide kernel's requests have more
  int nt;                                 // 16-row fragments of the other kernel
  bool split;                             // whether its items' tokens are split
  int groups;                             // into as many workgroups
  int wide_parts;
  int64_t few_bytes, wide_work;           // workspace of each (0: no split)
};

// Few items of few tokens are not split: a workgroup of eight waves an item.  Measured, 8
// cached heads and one query of 32, whole and split with the join (us):
//   requests x tokens  1 x 500     1 x 1000    1 x 2000    16 x 900    64 x 500   400 x 500
//   64 channels         7.4  10.5   9.6  10.5  13.9  10.5   9.8  12.8  10.4 15.1   61  43
//   128                 8.3  11.7  11.1  11.8  16.7  11.8  11.3  14.7  19.1 19.4  117  60
//   256                12.9  15.6  19.3  15.9  31.5  15.9  19.9  22.9  29.3 25.9  195 142
// The lines are drawn for 128 channels; for 256 they would be lower, by up to 3.4 us a call.
// Tiles have 16 rows there, else 32 if a request's rows fill them and the registers allow
// (128 channels): 24 rows over 500 tokens 9.3 us and with 32 16.8, but for 64 requests 35.9 and
// 21.7, which stay whole up to 256 tokens (of 100: 12.5 us, split 19.6).
constexpr int64_t kFewItems = 512, kFewTokens = 1024;
void plan_few(Plan &p, int64_t T, int64_t group, int64_t heads, int64_t D, int64_t B, int64_t rows,
              int64_t max_seq) {
  auto items = [&](int64_t tile) {
    return heads * std::min(B * up(rows, tile), up(T * group, tile) + B);
  };
  p.nt = 1;
  p.split = max_seq > kFewTokens || items(16) > kFewItems;
  if (p.split && D < 256 && rows > 16) {
    p.nt = 2;
    p.split = max_seq > 256 || items(32) > kFewItems;
  }
}

Plan plan_of(int64_t T, int64_t group, int64_t heads, int64_t D, int64_t B, int64_t max_query,
             int64_t max_seq, int64_t bytes) {
  Plan p = {};
  max_query = std::min(max_query, T);     // (so that no product below passes 64 bits)
  const int64_t items = wide_tiles(T, group, B) * heads;
  p.wide = max_query * group > kFewRows && items > 0 && items <= kMaxGrid;
  p.few = !p.wide || (T - (B - 1) * max_query) * group <= kFewRows;
  p.few_rows = p.few ? (p.wide ? kFewRows : INT32_MAX) : 0;
  const int64_t rows = max_query * group;
  plan_few(p, T, group, heads, D, B, p.wide && rows > kFewRows ? kFewRows : rows, max_seq);
  p.groups = split_groups(D, p.nt, B * heads, max_seq);
  p.few_bytes = p.few && p.split ? partial_bytes(D, p.nt, p.groups) : 0;
  p.wide_parts = 1;
  if (p.wide) {
    // Two workgroups a CU; a part is at least kLeastPart tokens (one request of 256 rows
    // over 2000 tokens 19 us, in parts of 128 tokens 20.3, of 512 25, of 1024 49).
    const int64_t room = 512 / items;
    const int64_t most = max_seq / kLeastPart;
    const int64_t parts = room < most ? room : most;
    p.wide_parts = (int)(parts < 1 ? 1 : (parts > 32 ? 32 : parts));
    p.wide_work = wide_bytes(items, p.wide_parts, D);
  }
  if (bytes >= 0 && bytes < p.few_bytes + p.wide_work) {
    p.few_bytes = p.wide_work = 0;
    p.wide_parts = 1;
  }
  return p;
}

}  // namespace

int64_t kv_attention_workspace(int64_t T, int64_t Hq, int64_t heads, int64_t D, int64_t B,
                               int64_t max_query, int64_t max_seq) {
  const Plan p = plan_of(T, Hq / heads, heads, D, B, max_query, max_seq, -1);
  return p.few_bytes + p.wide_work;
}

hipError_t launch_kv_attention(const AttentionArgs &args, int64_t D, int64_t max_query,
                               int64_t max_seq, float *workspace, int64_t workspace_bytes,
                               hipStream_t stream) {
  AttentionArgs a = args;
  const Plan p = plan_of(a.T, a.group, a.heads, D, a.B, max_query, max_seq, workspace_bytes);
  a.most_rows = p.few_rows;
  if (p.wide) {
    const hipError_t e = launch_kv_attention_wide(a, D, p.few_rows, p.wide_parts,
                                                  workspace + p.few_bytes / 4, stream);
    if (e != hipSuccess || !p.few) return e;
  }
  const unsigned groups = p.few_bytes > 0 ? p.groups : 0;        // (0: not split)
  auto run = [&](auto channels) {
    constexpr int kD = decltype(channels)::value;
    if constexpr (kD < 256)
      if (p.nt == 2) return launch<kD, 2, 4>(a, groups, workspace, stream);
    return groups ? launch<kD, 1, 4>(a, groups, workspace, stream)
                  : launch<kD, 1, 8>(a, groups, workspace, stream);
  };
  if (D == 64) return run(std::integral_constant<int, 64>{});
  if (D == 128) return run(std::integral_constant<int, 128>{});
  return run(std::integral_constant<int, 256>{});
}

}  // namespace rfq
