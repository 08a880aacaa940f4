// Router of a layer of experts: the k largest of each token's logits, their softmax
// weights, and the gradient.
//
// With S the chosen experts, m = max_i l_i and p_i = exp(l_i - m):
//     w_j = p_{S_j} / sum_{i in S} p_i   (renormalize)   or   / sum_i p_i,
//     dl_{S_j} = w_j (dw_j - s),  s = sum_j dw_j w_j, elsewhere 0   (renormalize)   or
//     dl_i = sum_{j: S_j = i} dw_j w_j - s p_i / sum p.
//
// A row of logits lies in the registers of kLanes lanes, R consecutive ones a lane: 16
// lanes (four rows a wave) up to 256 experts, the whole wave up to 1024.  A choice is the
// maximum of the lane's R and over the lanes, in DPP steps without LDS, then the lowest of the
// indices that reach it.  Logits are compared as integers of the same order, with NaN above
// all, so that infinities and what was taken (below -infinity, which is never chosen) need no
// case of their own.  A bf16 logit leaves room for its index in the same integer, the lower the
// larger: the maximum is then the choice itself.
//
// Bound by the instructions of the choices (5.5 R + 12 a choice for fp32, 2.5 R + 5 for bf16)
// and, for a softmax over all logits, by their exponentials.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts.h"
#include "gemm_common.h"

namespace rfq {
namespace {

constexpr int kThreads = 256;
constexpr int kTaken = INT32_MIN;              // below every key
constexpr int kNever = (int)0x807FFFFF;        // the key of -infinity

// Integers in the order of the floats: NaN above +infinity, -0 as +0.
__device__ __forceinline__ int order_of(float v) {
  if (v != v) return INT32_MAX;
  const int b = __float_as_int(v + 0.0f);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
// The key of logit `index`, and the value and (bf16) the index of a key.
template <bool BF16>
__device__ __forceinline__ int key_of(float v, int index) {
  return BF16 ? (order_of(v) & (int)0xFFFF0000) | (0xFFFF ^ index) : order_of(v);
}
template <bool BF16>
__device__ __forceinline__ float value_of(int key) {
  const int b = key ^ ((key >> 31) & 0x7FFFFFFF);
  return __int_as_float(BF16 ? b & (int)0xFFFF0000 : b);
}
__device__ __forceinline__ int index_of(int key) { return 0xFFFF ^ (key & 0xFFFF); }

// exp(x) for x <= 0 (and NaN): 2^(x log2 e) with the product's rounding error, which grows with
// |x|, multiplied back in.  Below -110, less than a float's least normal number, 0.
__device__ __forceinline__ float exp_of(float x) {
  x = x < -110.0f ? -110.0f : x;
  constexpr float kHi = 1.44269502162933349609f, kLo = 1.92596303e-8f;   // log2(e)
  const float h = x * kHi, l = fmaf(x, kHi, -h) + x * kLo;
  const float e = __builtin_amdgcn_exp2f(h);
  return fmaf(e * l, 0.693147182f, e);
}

// Combination of a lane's value with another's: all lanes of the row hold the result.
template <int kCtrl, class T>
__device__ __forceinline__ T from(T v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(i, i, kCtrl, 0xF, 0xF, false));
}
template <int kLanes, class T, class Op>
__device__ __forceinline__ T over_row(T v, Op op) {
  v = op(v, from<0xB1>(v));      // the neighbour in a pair
  v = op(v, from<0x4E>(v));      // the other pair of four
  v = op(v, from<0x141>(v));     // mirrored in eight
  v = op(v, from<0x140>(v));     // mirrored in sixteen
  if constexpr (kLanes == 64) {
    v = op(v, __shfl_xor(v, 16));
    v = op(v, __shfl_xor(v, 32));
  }
  return v;
}
struct Max { __device__ int operator()(int a, int b) const { return max(a, b); } };
struct Min { __device__ int operator()(int a, int b) const { return min(a, b); } };
struct Sum { __device__ float operator()(float a, float b) const { return a + b; } };

// Bytes of the loads that a lane's logits divide into.
constexpr int piece_bytes(int bytes) {
  return bytes % 16 == 0 ? 16 : (bytes % 8 == 0 ? 8 : (bytes % 4 == 0 ? 4 : 2));
}

// The lane's logits i0 .. i0 + R - 1 of a row (past E: -infinity) as keys.  VEC: E a multiple
// of R and rows at multiples of the lane's bytes (at most 16).
template <int R, bool BF16, bool VEC>
__device__ __forceinline__ void load_keys(const void *row, int i0, int E, int (&key)[R]) {
  if constexpr (VEC) {
    constexpr int kBytes = R * (BF16 ? 2 : 4), kPiece = piece_bytes(kBytes);
    constexpr int kPer = kPiece / (BF16 ? 2 : 4);
    if (i0 >= E) {
#pragma unroll
      for (int r = 0; r < R; ++r) key[r] = key_of<BF16>(-INFINITY, i0 + r);
      return;
    }
    const uint8_t *p = static_cast<const uint8_t *>(row) + (int64_t)i0 * (BF16 ? 2 : 4);
#pragma unroll
    for (int c = 0; c < kBytes / kPiece; ++c) {
      uint32_t w[4] = {0, 0, 0, 0};
      const uint8_t *at = p + kPiece * c;
      if constexpr (kPiece == 16) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(at);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else if constexpr (kPiece == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(at);
        w[0] = v.x; w[1] = v.y;
      } else if constexpr (kPiece == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(at);
      } else {
        w[0] = *reinterpret_cast<const uint16_t *>(at);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float f = BF16 ? __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16)
                             : __uint_as_float(w[i]);
        key[c * kPer + i] = key_of<BF16>(f, i0 + c * kPer + i);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = min(i0 + r, E - 1);
      const float f = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16)
                           : static_cast<const float *>(row)[i];
      key[r] = key_of<BF16>(i0 + r < E ? f : -INFINITY, i0 + r);
    }
  }
}

// sum of exp(l - m) over the row's logits; m their largest (where that is -infinity, NaN).
template <int kLanes, int R, bool BF16>
__device__ __forceinline__ float exp_sum(const int (&key)[R], float m) {
  float s = 0.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) s += exp_of(value_of<BF16>(key[r]) - m);
  return over_row<kLanes>(s, Sum{});
}

template <int kLanes, int R, bool BF16, bool VEC>
__global__ __launch_bounds__(kThreads) void route_kernel(const void *__restrict__ logits, int64_t T,
                                                         int E, int k, int renormalize,
                                                         float *__restrict__ weights,
                                                         int32_t *__restrict__ experts) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int lane = threadIdx.x % kLanes, i0 = lane * R;
  // (A row past the last is the last one again, so that no lane leaves the DPP steps.)
  const int64_t row = min(t, T - 1);
  int key[R];
  load_keys<R, BF16, VEC>(static_cast<const uint8_t *>(logits) + row * E * (BF16 ? 2 : 4), i0, E,
                          key);
  int left[R], mine = kNever, mine_at = -1, top = kNever;
  float total = 0.0f;
  for (int j = 0; j < k; ++j) {
    int best = key[0];
#pragma unroll
    for (int r = 1; r < R; ++r) best = max(best, key[r]);
    const int most = over_row<kLanes>(best, Max{});
    int where;
    if constexpr (BF16) {
      where = index_of(most);
#pragma unroll
      for (int r = 0; r < R; ++r) left[r] = key[r] == most ? kTaken : key[r];
    } else {
      int at = INT32_MAX;
#pragma unroll
      for (int r = R - 1; r >= 0; --r) at = key[r] == most ? i0 + r : at;
      where = over_row<kLanes>(at, Min{});
#pragma unroll
      for (int r = 0; r < R; ++r) left[r] = where - i0 == r ? kTaken : key[r];
    }
    if (j == 0) {
      top = most;
      if (!renormalize) total = exp_sum<kLanes, R, BF16>(key, value_of<BF16>(top));
    }
    if (lane == j) {
      mine = most;
      mine_at = most > kNever ? where : -1;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = left[r];
  }
  const float e = mine > kNever ? exp_of(value_of<BF16>(mine) - value_of<BF16>(top)) : 0.0f;
  if (renormalize) total = over_row<kLanes>(e, Sum{});
  if (t < T && lane < k) {
    weights[t * k + lane] = mine_at >= 0 ? e / total : 0.0f;
    experts[t * k + lane] = mine_at;
  }
}

template <int kLanes, int R, bool BF16, bool VEC>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(
    const float *__restrict__ dweights, const void *__restrict__ logits, int64_t T, int E, int k,
    const float *__restrict__ weights, const int32_t *__restrict__ experts, int renormalize,
    void *__restrict__ dlogits) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int lane = threadIdx.x % kLanes, i0 = lane * R;
  const int64_t row = min(t, T - 1);
  constexpr int kElem = BF16 ? 2 : 4;
  // Lane j holds choice j.
  const bool has = lane < k;
  const int64_t at = row * k + (has ? lane : 0);
  const int named = has ? experts[at] : -1, expert = (uint32_t)named < (uint32_t)E ? named : -1;
  const float w = has ? weights[at] : 0.0f;
  float g = expert >= 0 ? w * dweights[at] : 0.0f;
  const float s = over_row<kLanes>(g, Sum{});
  float d[R];
  if (renormalize) {
    if (expert >= 0) g -= w * s;
#pragma unroll
    for (int r = 0; r < R; ++r) d[r] = 0.0f;
  } else {
    int key[R];
    load_keys<R, BF16, VEC>(static_cast<const uint8_t *>(logits) + row * E * kElem, i0, E, key);
    int best = key[0];
#pragma unroll
    for (int r = 1; r < R; ++r) best = max(best, key[r]);
    const float top = value_of<BF16>(over_row<kLanes>(best, Max{}));
    const bool none = top == -INFINITY;
    const float m = none ? 0.0f : top;
    const float sum = exp_sum<kLanes, R, BF16>(key, m);
    const float per = none ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int r = 0; r < R; ++r)
      d[r] = -(exp_of(value_of<BF16>(key[r]) - m) * per) * s;
  }
  for (int j = 0; j < k; ++j) {
    const int i = __shfl(expert, j, kLanes);
    const float v = __shfl(g, j, kLanes);
#pragma unroll
    for (int r = 0; r < R; ++r) d[r] += i0 + r == i ? v : 0.0f;
  }
  if (t >= T) return;
  uint8_t *out = static_cast<uint8_t *>(dlogits) + (t * E + i0) * kElem;
  if constexpr (VEC) {
    if (i0 >= E) return;
    constexpr int kBytes = R * kElem, kPiece = piece_bytes(kBytes);
    uint32_t u[(kBytes + 3) / 4];
#pragma unroll
    for (int c = 0; c < (kBytes + 3) / 4; ++c) {
      if constexpr (BF16) u[c] = bf16x2_rne(d[2 * c], 2 * c + 1 < R ? d[(2 * c + 1) % R] : 0.0f);
      else u[c] = __float_as_uint(d[c]);
    }
#pragma unroll
    for (int c = 0; c < kBytes / kPiece; ++c) {
      uint8_t *at = out + kPiece * c;
      if constexpr (kPiece == 16)
        *reinterpret_cast<u32x4 *>(at) = u32x4{u[4 * c], u[4 * c + 1], u[4 * c + 2], u[4 * c + 3]};
      else if constexpr (kPiece == 8)
        *reinterpret_cast<uint2 *>(at) = make_uint2(u[2 * c], u[2 * c + 1]);
      else if constexpr (kPiece == 4)
        *reinterpret_cast<uint32_t *>(at) = u[c];
      else
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)(u[c / 2] >> (16 * (c & 1)));
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (i0 + r < E) {
        if constexpr (BF16) reinterpret_cast<uint16_t *>(out)[r] = (uint16_t)bf16_rne(d[r]);
        else reinterpret_cast<float *>(out)[r] = d[r];
      }
    }
  }
}

// Calls go(shape) with the shape that holds E logits.  Where E is not a multiple of its R, logits
// are loaded and gradients stored one by one (vector_rows()).  32768 tokens, 6 choices, softmax over
// all, us, fp32 | bf16:             E =    80          144         176
//   route                            8.3 | 6.7   10.8 | 8.9  12.2 | 10.0
//   route in the next shape          8.8 | 6.8   10.7 | 8.3  12.9 |  9.8
//   gradient                        10.4 | 7.6   20.6 | 13.0 28.7 | 17.0
//   gradient in the next shape       8.4 | 8.0   10.8 | 10.6 15.2 | 12.0
template <int L, int N>
struct Shape {
  static constexpr int kLanes = L, R = N;
};
template <class Go>
hipError_t on_shape(int E, Go go) {
  if (E <= 16) return go(Shape<16, 1>{});
  if (E <= 32) return go(Shape<16, 2>{});
  if (E <= 64) return go(Shape<16, 4>{});
  if (E <= 96) return go(Shape<16, 6>{});
  if (E <= 128) return go(Shape<16, 8>{});
  if (E <= 160) return go(Shape<16, 10>{});
  if (E <= 192) return go(Shape<16, 12>{});
  if (E <= 256) return go(Shape<16, 16>{});
  if (E <= 512) return go(Shape<64, 8>{});
  return go(Shape<64, 16>{});
}

// Rows start at multiples of a lane's bytes (16 at most), and no lane's logits end
// inside a row.
template <int R>
bool vector_rows(const void *a, const void *b, int E, bool bf16) {
  const int piece = piece_bytes(R * (bf16 ? 2 : 4));
  const uintptr_t p = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b);
  return E % R == 0 && p % piece == 0;
}

}  // namespace

hipError_t launch_route(const void *logits, bool bf16, int64_t T, int E, int k, bool renormalize,
                        float *weights, int32_t *experts, hipStream_t stream) {
  return on_shape(E, [&](auto shape) {
    constexpr int kLanes = decltype(shape)::kLanes, R = decltype(shape)::R;
    const dim3 grid((unsigned)((T + kThreads / kLanes - 1) / (kThreads / kLanes)));
    const bool vec = vector_rows<R>(logits, nullptr, E, bf16);
    auto kern = bf16 ? (vec ? route_kernel<kLanes, R, true, true> : route_kernel<kLanes, R, true, false>)
                     : (vec ? route_kernel<kLanes, R, false, true> : route_kernel<kLanes, R, false, false>);
    kern<<<grid, kThreads, 0, stream>>>(logits, T, E, k, renormalize, weights, experts);
    return hipGetLastError();
  });
}

hipError_t launch_route_backward(const float *dweights, const void *logits, bool bf16, int64_t T,
                                 int E, int k, const float *weights, const int32_t *experts,
                                 bool renormalize, void *dlogits, hipStream_t stream) {
  return on_shape(E, [&](auto shape) {
    constexpr int kLanes = decltype(shape)::kLanes, R = decltype(shape)::R;
    const dim3 grid((unsigned)((T + kThreads / kLanes - 1) / (kThreads / kLanes)));
    const bool vec = vector_rows<R>(logits, dlogits, E, bf16);
    auto kern = bf16 ? (vec ? route_backward_kernel<kLanes, R, true, true>
                            : route_backward_kernel<kLanes, R, true, false>)
                     : (vec ? route_backward_kernel<kLanes, R, false, true>
                            : route_backward_kernel<kLanes, R, false, false>);
    kern<<<grid, kThreads, 0, stream>>>(dweights, logits, T, E, k, weights, experts, renormalize,
                                        dlogits);
    return hipGetLastError();
  });
}

}  // namespace rfq
