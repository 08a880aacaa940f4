// Router of a layer of experts: the k largest of each token's logits, their softmax
// weights, and the gradient.
//
// With S the chosen experts, m = max_i l_i and p_i = exp(l_i - m):
//     w_j = p_{S_j} / sum_{i in S} p_i   (renormalize)   or   / sum_i p_i,
//     dl_{S_j} = w_j (dw_j - s),  s = sum_j dw_j w_j, elsewhere 0   (renormalize)   or
//     dl_i = sum_{j: S_j = i} dw_j w_j - s p_i / sum p.
//
// A row of logits lies in the registers of kLanes lanes, R consecutive ones a lane: 16
// lanes (four rows a wave) up to 256 experts, the whole wave up to 1024.  A choice is a
// scan of the lane's R, a maximum over the lanes and a minimum over the indices of those
// that reach it (ties go to the lowest index), in DPP steps without LDS.  Logits are compared
// as integers of the same order, with NaN above all, so that infinities and what was taken
// (below -infinity, which is never chosen) need no case of their own.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts.h"
#include "gemm_common.h"

namespace rfq {
namespace {

constexpr int kThreads = 256;
constexpr int kTaken = INT32_MIN;              // below every logit's key
constexpr int kNever = (int)0x807FFFFF;        // the key of -infinity

// Integers in the order of the floats: NaN above +infinity, -0 as +0.
__device__ __forceinline__ int key_of(float v) {
  if (v != v) return INT32_MAX;
  const int b = __float_as_int(v + 0.0f);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float value_of(int key) {
  return __int_as_float(key ^ ((key >> 31) & 0x7FFFFFFF));
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

// The lane's logits i0 .. i0 + R - 1 of a row (past E: kTaken) as keys.  VEC: E a multiple
// of R and rows at multiples of the lane's bytes (at most 16).
template <int R, bool BF16, bool VEC>
__device__ __forceinline__ void load_keys(const void *row, int i0, int E, int (&key)[R]) {
  if constexpr (VEC) {
    constexpr int kBytes = R * (BF16 ? 2 : 4), kPiece = kBytes < 16 ? kBytes : 16;
    constexpr int kPer = kPiece / (BF16 ? 2 : 4);
    if (i0 >= E) {
#pragma unroll
      for (int r = 0; r < R; ++r) key[r] = kTaken;
      return;
    }
    const uint8_t *p = static_cast<const uint8_t *>(row) + (int64_t)i0 * (BF16 ? 2 : 4);
#pragma unroll
    for (int c = 0; c < kBytes / kPiece; ++c) {
      uint32_t w[4] = {0, 0, 0, 0};
      if constexpr (kPiece == 16) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(p + 16 * c);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else if constexpr (kPiece == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        w[0] = v.x; w[1] = v.y;
      } else if constexpr (kPiece == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
      } else {
        w[0] = *reinterpret_cast<const uint16_t *>(p);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float f = BF16 ? __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16)
                             : __uint_as_float(w[i]);
        key[c * kPer + i] = key_of(f);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = min(i0 + r, E - 1);
      const float f = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16)
                           : static_cast<const float *>(row)[i];
      key[r] = i0 + r < E ? key_of(f) : kTaken;
    }
  }
}

// sum of exp(l - m) over the row's logits (0 where all are -infinity; m is then unused).
template <int kLanes, int R>
__device__ __forceinline__ float exp_sum(const int (&key)[R], float m) {
  float s = 0.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) s += key[r] > kNever ? expf(value_of(key[r]) - m) : 0.0f;
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
  int mine = kNever, mine_at = -1, top = kNever;
  float total = 0.0f;
  for (int j = 0; j < k; ++j) {
    int best = key[0], at = i0;
#pragma unroll
    for (int r = 1; r < R; ++r) {
      at = key[r] > best ? i0 + r : at;
      best = max(best, key[r]);
    }
    const int most = over_row<kLanes>(best, Max{});
    const int where = over_row<kLanes>(best == most ? at : INT32_MAX, Min{});
    if (j == 0) {
      top = most;
      if (!renormalize) total = exp_sum<kLanes, R>(key, value_of(top));
    }
    if (lane == j) {
      mine = most;
      mine_at = most > kNever ? where : -1;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = i0 + r == where ? kTaken : key[r];
  }
  const float e = mine > kNever ? expf(value_of(mine) - value_of(top)) : 0.0f;
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
    const float m = value_of(over_row<kLanes>(best, Max{}));
    const float total = exp_sum<kLanes, R>(key, m);
#pragma unroll
    for (int r = 0; r < R; ++r)
      d[r] = key[r] > kNever ? -(expf(value_of(key[r]) - m) / total) * s : 0.0f;
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
    uint32_t u[(R * kElem + 3) / 4];
#pragma unroll
    for (int c = 0; c < (R * kElem + 3) / 4; ++c) {
      if constexpr (BF16) u[c] = bf16x2_rne(d[2 * c], R > 1 ? d[(2 * c + 1) % R] : 0.0f);
      else u[c] = __float_as_uint(d[c]);
    }
    constexpr int kBytes = R * kElem;
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int c = 0; c < kBytes / 16; ++c)
        reinterpret_cast<u32x4 *>(out)[c] = u32x4{u[4 * c], u[4 * c + 1], u[4 * c + 2], u[4 * c + 3]};
    } else if constexpr (kBytes == 8) {
      *reinterpret_cast<uint2 *>(out) = make_uint2(u[0], u[1]);
    } else if constexpr (kBytes == 4) {
      *reinterpret_cast<uint32_t *>(out) = u[0];
    } else {
      *reinterpret_cast<uint16_t *>(out) = (uint16_t)u[0];
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

// Calls go(shape) with the shape that holds E logits.
template <int L, int N>
struct Shape {
  static constexpr int kLanes = L, R = N;
};
template <class Go>
hipError_t on_shape(int E, Go go) {
  if (E <= 16) return go(Shape<16, 1>{});
  if (E <= 32) return go(Shape<16, 2>{});
  if (E <= 64) return go(Shape<16, 4>{});
  if (E <= 128) return go(Shape<16, 8>{});
  if (E <= 256) return go(Shape<16, 16>{});
  if (E <= 512) return go(Shape<64, 8>{});
  return go(Shape<64, 16>{});
}

// Rows start at multiples of a lane's bytes (16 at most), and no lane's logits end
// inside a row.
template <int R>
bool vector_rows(const void *a, const void *b, int E, bool bf16) {
  const int bytes = R * (bf16 ? 2 : 4), piece = bytes < 16 ? bytes : 16;
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
