// Device code shared by the attention kernels over the MXFP4 key/value cache:
// decoding to bf16, exchanges between lanes, the transposing LDS read and a request's
// extent.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv.h"
#include "mx_device.h"

namespace rfq {
namespace {

constexpr float kLn2 = 0.69314718055994531f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float across_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float across_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ uint32_t c_byte(uint32_t w, int i) { return w >> (8 * i) & 0xFFu; }

// Lane `from`'s value in every lane (a scalar).
__device__ __forceinline__ int64_t lane_value(int64_t v, int from) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, from) |
         (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), from) << 32;
}

// 8 codes to bf16 times their block's scale.
__device__ __forceinline__ u32x4 decode_bf16(uint32_t c, float s) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return r;
}

// Orders a wave's LDS accesses (the memory serves them in order).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ v4f mma(const u32x4 &a, const u32x4 &b, const v4f &c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Element i of lane l: 16-bit element (l mod 16) of row 4 (l / 16) + i, each lane
// pointing at 4 elements: lanes 4 j .. 4 j + 3 of a group of 16 at its row j.
__device__ __forceinline__ u32x2 read_transposed(const uint8_t *p) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// A request's rows and tokens.  S: a kernel's shape.
struct Request {
  int start, nq, len;
  int tiles0, tiles;                      // first token tile that a row sees; number (>= 1)
  int row_tiles;
};

template <class S>
__device__ __forceinline__ Request request(const AttentionArgs &a, int start, int nq, int len) {
  Request r = {start, nq, len};
  int first = 0;
  if (a.window) first = max(0, len - nq - a.window + 1);
  r.tiles0 = min(first, len) / S::kTile;
  r.tiles = max(1, (len + S::kTile - 1) / S::kTile - r.tiles0);
  r.row_tiles = (nq * a.group + S::kRows - 1) / S::kRows;
  return r;
}
template <class S>
__device__ __forceinline__ Request request(const AttentionArgs &a, int b) {
  const int s0 = min(max(a.starts[b], 0), a.T), s1 = min(max(a.starts[b + 1], s0), a.T);
  return request<S>(a, s0, s1 - s0, min(max(a.lens[b], 0), a.capacity));
}

}  // namespace
}  // namespace rfq
