// Rotary positions with several axes, and the key/value cache's write and
// read-back.
//
// A pair (a, b) of a head's channels turns by the angle of its own position axis:
// (a c - b s, b c + a s), the gradient by the opposite angle (s -> -s).  Cosines and
// sines come from a table [position][pair] that the program makes once, in whatever
// precision: no angle is formed here, so a position of any size costs the same and
// loses nothing.  Products and sums are rounded one by one (no fused multiply-add),
// which makes the rotated values, and the 4-bit codes made from them, the same
// wherever they are computed in fp32.
//
// Everything here streams: an element is read and written once and a few
// operations are done on it.  A workgroup takes one token, or in rfq_rope a few
// (all heads share a token's angles); the angles of its pairs, each with its own
// axis and so its own table row, are fetched once by one thread a pair into LDS, and
// every head's threads read them from there.  The elements' own loads are issued
// before that and arrive under it.  Threads hold 8 + 8 channels of a head:
// the two halves that turn together, or 16 neighbours where the pairs are neighbours
// or the channels are copied.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv.h"
#include "mx_device.h"
#include "rfq_internal.h"

namespace rfq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// What the kernels need of rfq_rope_spec (axes by value: host memory).
struct Rope {
  const int32_t *positions;
  int64_t positions_stride;
  const float2 *cos_sin;
  int32_t max_pos, half, interleaved;
  float sign;
  uint8_t axes[kMaxPairs];
};

// n / d for n < 2^24, d <= 2^12: m = ceil(2^32 / d).
struct Divider {
  uint32_t d, m;
};
__device__ __forceinline__ uint32_t divided(uint32_t n, const Divider &v) {
  return v.d == 1 ? n : __umulhi(n, v.m);
}
Divider divider(uint32_t d) { return {d, (uint32_t)(((uint64_t(1) << 32) + d - 1) / d)}; }

// The angle of pair j of token t: (cos, +-sin), NaN where the position is outside
// the table.
__device__ __forceinline__ float2 angle(const Rope &r, int64_t t, int j) {
  const int32_t p = r.positions[r.axes[j] * r.positions_stride + t];
  float2 cs = make_float2(__builtin_nanf(""), __builtin_nanf(""));
  if (p >= 0 && p < r.max_pos) cs = r.cos_sin[(int64_t)p * r.half + j];
  cs.y *= r.sign;
  return cs;
}

// 8 consecutive elements.
template <bool BF16>
struct Piece {
  u32x4 w[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Piece<BF16> load8(const void *base, int64_t at) {
  Piece<BF16> p;
  const u32x4 *s = reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(base) +
                                                   at * (BF16 ? 2 : 4));
  p.w[0] = s[0];
  if constexpr (!BF16) p.w[1] = s[1];
  return p;
}
template <bool BF16>
__device__ __forceinline__ void store8(void *base, int64_t at, const Piece<BF16> &p) {
  u32x4 *d = reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(base) + at * (BF16 ? 2 : 4));
  d[0] = p.w[0];
  if constexpr (!BF16) d[1] = p.w[1];
}
template <bool BF16>
__device__ __forceinline__ f32x8 values(const Piece<BF16> &p) {
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (BF16)
      v[i] = __uint_as_float(i & 1 ? p.w[0][i / 2] & 0xFFFF0000u : p.w[0][i / 2] << 16);
    else
      v[i] = __uint_as_float(p.w[i / 4][i % 4]);
  }
  return v;
}
// Rounded once, to nearest even.
template <bool BF16>
__device__ __forceinline__ Piece<BF16> rounded(const f32x8 &v) {
  Piece<BF16> p;
  if constexpr (BF16) {
    p.w[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p.w[i / 4][i % 4] = __float_as_uint(v[i]);
  }
  return p;
}

__device__ __forceinline__ void turn(float &a, float &b, float2 cs) {
#pragma clang fp contract(off)
  const float x = a * cs.x - b * cs.y;
  b = b * cs.x + a * cs.y;
  a = x;
}
// a[i], b[i] as pairs (i), or with interleaved a and then b as neighbouring ones.
__device__ __forceinline__ void turn8(f32x8 &a, f32x8 &b, const float2 *cs, bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float x = a[i], y = a[i + 1], z = b[i], w = b[i + 1];
      turn(x, y, cs[i / 2]);
      turn(z, w, cs[4 + i / 2]);
      a[i] = x; a[i + 1] = y; b[i] = z; b[i + 1] = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x = a[i], y = b[i];
      turn(x, y, cs[i]);
      a[i] = x; b[i] = y;
    }
  }
}

// Unit u of a head (16 channels): where its two pieces are, and its first pair
// (-1: channels that are copied).
struct Unit {
  int c0, c1, pair;
};
__device__ __forceinline__ Unit unit_of(int u, int half, bool interleaved) {
  if (u >= half / 8) return {16 * u, 16 * u + 8, -1};
  return interleaved ? Unit{16 * u, 16 * u + 8, 8 * u} : Unit{8 * u, half + 8 * u, 8 * u};
}

// y = rotated x.  A workgroup takes `tokens` tokens; thread = (token, head lane,
// unit), stepping over the heads four at a time so that four heads' loads are in
// flight.  Bandwidth bounds it: 32768 tokens of 40 heads of 128 channels (bf16, three
// axes, the gradient's direction) in 131 us, 5.1 TB/s read and written, which is what
// a large copy reaches on the card; 1000 tokens of 40 heads take 5.6 us.
constexpr int kRopeBatch = 4;
template <bool BF16>
__global__ __launch_bounds__(kThreads) void rope_kernel(const uint8_t *x, int64_t x_ts,
                                                        int64_t x_hs, uint8_t *y, int64_t y_ts,
                                                        int64_t y_hs, int64_t T, int H, int units,
                                                        int head_lanes, int tokens,
                                                        const Rope rope) {
  extern __shared__ float2 angles[];              // [tokens][half]
  const int half = rope.half;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int per_token = units * head_lanes;
  const int tok = threadIdx.x / per_token, r = threadIdx.x - tok * per_token;
  const int lane_h = r / units, u = r - lane_h * units;
  const int64_t t = t0 + tok;
  const bool mine = tok < tokens && t < T;
  const Unit un = unit_of(u, half, rope.interleaved);
  const uint8_t *xb = x + (mine ? t * x_ts : 0) * (BF16 ? 2 : 4);
  uint8_t *yb = y + (mine ? t * y_ts : 0) * (BF16 ? 2 : 4);

  Piece<BF16> a[kRopeBatch], b[kRopeBatch];
  auto fetch = [&](int h) {
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int hi = h + i * head_lanes;
      if (mine && hi < H) {
        a[i] = load8<BF16>(xb, hi * x_hs + un.c0);
        b[i] = load8<BF16>(xb, hi * x_hs + un.c1);
      }
    }
  };
  fetch(lane_h);
  for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
    const int k = i / half;
    if (t0 + k < T) angles[i] = angle(rope, t0 + k, i - k * half);
  }
  __syncthreads();
  float2 cs[8];
  if (un.pair >= 0 && mine) {
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = angles[tok * half + un.pair + i];
  }
  for (int h = lane_h; mine && h < H; h += kRopeBatch * head_lanes) {
    if (h != lane_h) fetch(h);
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int hi = h + i * head_lanes;
      if (hi >= H) break;
      if (un.pair >= 0) {
        f32x8 va = values<BF16>(a[i]), vb = values<BF16>(b[i]);
        turn8(va, vb, cs, rope.interleaved);
        a[i] = rounded<BF16>(va);
        b[i] = rounded<BF16>(vb);
      }
      store8<BF16>(yb, hi * y_hs + un.c0, a[i]);
      store8<BF16>(yb, hi * y_hs + un.c1, b[i]);
    }
  }
}

// The largest magnitude's bits over the 4 lanes of a block (as integers: infinities
// and NaN are the largest).
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);
  v = a > v ? a : v;
  const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);
  return b > v ? b : v;
}

// MXFP4 of 8 values of a block whose other values are in the lanes of the quad:
// codes and scale byte (0xFF and no codes for a block that is not finite).
__device__ __forceinline__ uint32_t quantize8(const f32x8 &v, uint32_t &byte) {
  uint32_t top = 0;
  float e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    e[i] = v[i];
    const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
    top = m > top ? m : top;
  }
  top = quad_max(top);
  const bool finite = top < 0x7F800000u;
  byte = finite ? scale_byte(__uint_as_float(top)) : 0xFFu;
  const uint32_t c = encode8(e, scale_operand(finite ? byte : 127u));
  return finite ? c : 0u;
}

struct Cache {
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int32_t heads, page_shift, D;
  int64_t slots;                                  // blocks * page
};

// Row (block, head, token) of a slot.
__device__ __forceinline__ int64_t row_of(const Cache &c, int slot, int head) {
  const int64_t block = slot >> c.page_shift;
  return ((block * c.heads + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}

struct Heads {
  const uint8_t *data;
  int64_t ts, hs;
};

// One token of a step.  Bandwidth bounds a large step: 8192 tokens, 32 heads of q and 8 of
// k and v of 128 channels (bf16), 177 MB in 33 us, 5.4 TB/s where a large copy reaches 5.1.
// 16 tokens take 3.4 us: the launch and the position's, the angle's and the value's way.
//
// Work items of a token: the units of q (16 channels), then
// the 8-channel pieces of k, then those of v, each class rounded up to whole waves;
// a workgroup takes 256 of them.  A quad of lanes holds a 32-channel block of k
// or v, so that its maximum is two exchanges within the quad; a piece of k also
// loads the piece that it turns with (from the cache lines its neighbours read).
template <bool BF16>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(
    Heads q, Heads k, Heads v, uint8_t *q_out, int64_t qo_ts, int64_t qo_hs,
    const int32_t *__restrict__ slots, const Cache cache, int q_items, int q_span, int kv_items,
    int kv_span, Divider q_units, Divider pieces, int has_rope, const Rope rope) {
  __shared__ float2 angles[kMaxPairs];
  const int64_t t = blockIdx.x;
  const int item = blockIdx.y * kThreads + threadIdx.x;
  const int half = has_rope ? rope.half : 0;
  const bool inter = rope.interleaved;
  // 0: q, 1: k, 2: v, 3: nothing.
  int role = 3, head = 0, c0 = 0, c1 = 0, pair = -1;
  bool first = true;                              // k: the piece holds the pairs' a
  const uint8_t *src = nullptr;
  if (item < q_span) {
    if (item < q_items) {
      head = divided(item, q_units);
      const Unit un = unit_of(item - head * q_units.d, half, inter);
      role = 0; c0 = un.c0; c1 = un.c1; pair = un.pair;
      src = q.data + (t * q.ts + head * q.hs) * (BF16 ? 2 : 4);
    }
  } else {
    int i = item - q_span;
    const bool is_v = i >= kv_span;
    i -= is_v ? kv_span : 0;
    if (i < kv_items) {
      head = divided(i, pieces);
      c0 = c1 = 8 * (i - head * (int)pieces.d);
      role = is_v ? 2 : 1;
      if (!is_v && c0 < 2 * half) {
        first = inter || c0 < half;
        pair = inter ? c0 / 2 : (first ? c0 : c0 - half);
        if (!inter) c1 = first ? c0 + half : c0 - half;
      }
      src = (is_v ? v.data : k.data) + (t * (is_v ? v.ts : k.ts) + head * (is_v ? v.hs : k.hs)) *
                                           (BF16 ? 2 : 4);
    }
  }
  Piece<BF16> a{}, b{};
  if (role != 3) {
    a = load8<BF16>(src, c0);
    if (c1 != c0) b = load8<BF16>(src, c1);
  }
  const int slot = slots[t];
  if (half) {
    for (int j = threadIdx.x; j < half; j += kThreads) angles[j] = angle(rope, t, j);
    __syncthreads();
  }
  if (role == 3) return;
  if (role == 0) {
    if (pair >= 0) {
      f32x8 va = values<BF16>(a), vb = values<BF16>(b);
      turn8(va, vb, angles + pair, inter);
      a = rounded<BF16>(va);
      b = rounded<BF16>(vb);
    }
    const int64_t at = t * qo_ts + head * qo_hs;
    store8<BF16>(q_out, at + c0, a);
    store8<BF16>(q_out, at + c1, b);
    return;
  }
  if (slot < 0 || slot >= cache.slots) return;    // the same for the whole token
  f32x8 val = values<BF16>(a);
  if (pair >= 0) {
    if (inter) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float x = val[i], y = val[i + 1];
        turn(x, y, angles[pair + i / 2]);
        val[i] = x; val[i + 1] = y;
      }
    } else {
      const f32x8 other = values<BF16>(b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x = first ? val[i] : other[i], y = first ? other[i] : val[i];
        turn(x, y, angles[pair + i]);
        val[i] = first ? x : y;
      }
    }
  }
  uint32_t byte;
  const uint32_t codes = quantize8(val, byte);
  const int64_t row = row_of(cache, slot, head);
  uint8_t *dc = role == 1 ? cache.k_codes : cache.v_codes;
  uint8_t *ds = role == 1 ? cache.k_scales : cache.v_scales;
  *reinterpret_cast<uint32_t *>(dc + row * (cache.D / 2) + c0 / 2) = codes;
  if ((threadIdx.x & 3) == 0) ds[row * (cache.D / 32) + c0 / 32] = (uint8_t)byte;
}

// 8 channels of one (slot, k or v, head) a thread.  Bandwidth bounds it, four bytes written
// for one read: 8192 slots of 8 heads of 128 channels to bf16, 42 MB, in 10.8 us; 16 in 2.6.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void kv_gather_kernel(const Cache cache,
                                                             const int32_t *__restrict__ slots,
                                                             int items, Divider pieces,
                                                             uint8_t *k_out, uint8_t *v_out) {
  const int64_t n = blockIdx.x;
  const int i = blockIdx.y * kThreads + threadIdx.x;
  if (i >= 2 * items) return;
  const bool is_v = i >= items;
  const int j = is_v ? i - items : i;
  const int head = divided(j, pieces), c0 = 8 * (j - head * (int)pieces.d);
  const int slot = slots[n];
  f32x8 v = {};
  if (slot >= 0 && slot < cache.slots) {
    const int64_t row = row_of(cache, slot, head);
    const uint8_t *dc = is_v ? cache.v_codes : cache.k_codes;
    const uint8_t *ds = is_v ? cache.v_scales : cache.k_scales;
    const uint32_t byte = ds[row * (cache.D / 32) + c0 / 32];
    float d[8];
    decode8(*reinterpret_cast<const uint32_t *>(dc + row * (cache.D / 2) + c0 / 2),
            scale_operand(byte), d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = byte == 0xFFu ? __builtin_nanf("") : d[e];
  }
  store8<BF16>(is_v ? v_out : k_out, (n * cache.heads + head) * cache.D + c0, rounded<BF16>(v));
}

Rope device_rope(const rfq_rope_spec &s, bool backward) {
  Rope r = {};
  r.positions = s.positions;
  r.positions_stride = s.positions_stride;
  r.cos_sin = reinterpret_cast<const float2 *>(s.cos_sin);
  r.max_pos = (int32_t)(s.max_pos < INT32_MAX ? s.max_pos : INT32_MAX);
  r.half = s.rotary / 2;
  r.interleaved = s.interleaved != 0;
  r.sign = backward ? -1.0f : 1.0f;
  for (int j = 0; j < r.half; ++j) r.axes[j] = s.axes ? s.axes[j] : 0;
  return r;
}

Cache device_cache(const rfq_kv_cache &c) {
  return {c.k_codes, c.k_scales, c.v_codes, c.v_scales, (int32_t)c.heads,
          __builtin_ctz((unsigned)c.page), (int32_t)c.D, c.blocks * c.page};
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

hipError_t launch_rope(const rfq_heads &x, bool bf16, int64_t T, int64_t H, int64_t D,
                       const rfq_rope_spec &rope, bool backward, const rfq_heads &y,
                       hipStream_t stream) {
  const int units = (int)(D / 16), slots = kThreads / units;
  // Few tokens: one a workgroup and as many heads side by side as fit.  From
  // kManyTokens on a token's threads take several heads each (8 lanes of heads) and its
  // angles serve more of them.  Measured, side by side and in 8 lanes: 256 tokens of 128
  // heads 5.3 and 8.5 us, 1024 of 128 13.1 and 14.8, 1024 of 40 equal; 2048 of 40 10.1 and
  // 8.9, 4096 of 40 18.4 and 15.5, 32768 of 24 96 and 82, of 128 equal.
  constexpr int64_t kManyTokens = 2048;
  const int most = (int)(H < slots ? H : slots);
  const int head_lanes = T >= kManyTokens && most > 8 ? 8 : most;
  const int tokens = slots / head_lanes;
  const Rope r = device_rope(rope, backward);
  const unsigned grid = (unsigned)up(T, tokens);
  const size_t lds = sizeof(float2) * (size_t)tokens * r.half;
  auto xb = static_cast<const uint8_t *>(x.data);
  auto yb = static_cast<uint8_t *>(y.data);
  if (bf16)
    rope_kernel<true><<<grid, kThreads, lds, stream>>>(xb, x.token_stride, x.head_stride, yb,
                                                       y.token_stride, y.head_stride, T, (int)H,
                                                       units, head_lanes, tokens, r);
  else
    rope_kernel<false><<<grid, kThreads, lds, stream>>>(xb, x.token_stride, x.head_stride, yb,
                                                        y.token_stride, y.head_stride, T, (int)H,
                                                        units, head_lanes, tokens, r);
  return hipGetLastError();
}

hipError_t launch_kv_append(const rfq_heads &k, const rfq_heads &v, bool bf16, int64_t T,
                            const int32_t *slots, const rfq_kv_cache &cache, const rfq_heads *q,
                            int64_t Hq, const rfq_rope_spec *rope, const rfq_heads *q_out,
                            hipStream_t stream) {
  const int D = (int)cache.D;
  const int q_items = q ? (int)Hq * (D / 16) : 0, kv_items = (int)cache.heads * (D / 8);
  const int q_span = (int)up(q_items, 64) * 64, kv_span = (int)up(kv_items, 64) * 64;
  auto heads = [](const rfq_heads &h) {
    return Heads{static_cast<const uint8_t *>(h.data), h.token_stride, h.head_stride};
  };
  const Heads hq = q ? heads(*q) : Heads{};
  uint8_t *qo = q ? static_cast<uint8_t *>(q_out->data) : nullptr;
  const int64_t qo_ts = q ? q_out->token_stride : 0, qo_hs = q ? q_out->head_stride : 0;
  const Rope r = rope ? device_rope(*rope, false) : Rope{};
  const dim3 grid((unsigned)T, (unsigned)up(q_span + 2 * kv_span, kThreads));
  if (bf16)
    kv_append_kernel<true><<<grid, kThreads, 0, stream>>>(
        hq, heads(k), heads(v), qo, qo_ts, qo_hs, slots, device_cache(cache), q_items, q_span,
        kv_items, kv_span, divider(D / 16), divider(D / 8), rope != nullptr, r);
  else
    kv_append_kernel<false><<<grid, kThreads, 0, stream>>>(
        hq, heads(k), heads(v), qo, qo_ts, qo_hs, slots, device_cache(cache), q_items, q_span,
        kv_items, kv_span, divider(D / 16), divider(D / 8), rope != nullptr, r);
  return hipGetLastError();
}

hipError_t launch_kv_gather(const rfq_kv_cache &cache, const int32_t *slots, int64_t n,
                            void *k_out, void *v_out, bool bf16, hipStream_t stream) {
  const int items = (int)(cache.heads * (cache.D / 8));
  const dim3 grid((unsigned)n, (unsigned)up(2 * items, kThreads));
  auto ko = static_cast<uint8_t *>(k_out);
  auto vo = static_cast<uint8_t *>(v_out);
  const Divider pieces = divider((uint32_t)(cache.D / 8));
  if (bf16)
    kv_gather_kernel<true><<<grid, kThreads, 0, stream>>>(device_cache(cache), slots, items,
                                                          pieces, ko, vo);
  else
    kv_gather_kernel<false><<<grid, kThreads, 0, stream>>>(device_cache(cache), slots, items,
                                                           pieces, ko, vo);
  return hipGetLastError();
}

}  // namespace rfq
