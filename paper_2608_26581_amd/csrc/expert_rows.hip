// The way of a layer's rows to the experts and back, and its gradients:
//     gather    xs[slots[t][j]] = x[t],  xs[s] = 0 where rows[s] is no row
//     combine   out[t] = sum_j w[t][j] z[slots[t][j]] (slots that are none: nothing)
//     backward  dz[slots[t][j]] = w[t][j] dout[t],  dw[t][j] = dout[t] . z[slots[t][j]],
//               dz[s] = 0 where rows[s] is no row.
// The gradient of gather is combine with weights of one.
//
// All are bound by memory: every element is read and written once, 16 bytes a lane where
// rows are whole multiples of 16 bytes.  Sums are fp32, in the order of j and, for dw, in a
// fixed tree over the row; no atomics.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "experts.h"
#include "gemm_common.h"

namespace rfq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// V consecutive elements (16 bytes, or one element) as fp32.
template <bool BF16, bool VEC>
struct Piece {
  static constexpr int kElem = BF16 ? 2 : 4;
  static constexpr int V = VEC ? 16 / kElem : 1;
  using Raw = std::conditional_t<VEC, u32x4, std::conditional_t<BF16, uint16_t, uint32_t>>;
  static __device__ __forceinline__ Raw load(const void *p, int64_t i) {
    return static_cast<const Raw *>(p)[i];
  }
  static __device__ __forceinline__ void store(void *p, int64_t i, Raw v) {
    static_cast<Raw *>(p)[i] = v;
  }
  static __device__ __forceinline__ void widen(Raw r, float (&f)[V]) {
    if constexpr (!VEC) {
      f[0] = __uint_as_float(BF16 ? (uint32_t)r << 16 : (uint32_t)r);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
          f[2 * i] = __uint_as_float(r[i] << 16);
          f[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        } else {
          f[i] = __uint_as_float(r[i]);
        }
      }
    }
  }
  static __device__ __forceinline__ Raw narrow(const float (&f)[V]) {
    if constexpr (!VEC) {
      if constexpr (BF16) return (Raw)bf16_rne(f[0]);
      else return (Raw)__float_as_uint(f[0]);
    } else {
      u32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) r[i] = bf16x2_rne(f[2 * i], f[2 * i + 1]);
        else r[i] = __float_as_uint(f[i]);
      }
      return r;
    }
  }
};

// A wave's part of a row: kPieces pieces a lane, `parts` of them a row.
constexpr int kPieces = 4;

// Row and part of a wave's work item (numbered in 32 bits), parts first.
struct Item { int64_t row; int part; };
__device__ __forceinline__ bool item_of(int64_t rows, int parts, Item &it) {
  const uint32_t w = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  it.row = w / (uint32_t)parts;
  it.part = (int)(w - (uint32_t)it.row * (uint32_t)parts);
  return it.row < rows;
}

// Zeros in the rows of y that are no token's, among the 64 slots from s0 on (a workgroup).
template <bool BF16, bool VEC>
__device__ __forceinline__ void clear_rows(const int32_t *rows, int64_t s0, int64_t P, int64_t T,
                                           int pieces, void *y) {
  using Q = Piece<BF16, VEC>;
  const int lane = threadIdx.x & 63;
  const int64_t r = s0 + lane < P ? rows[s0 + lane] : 0;
  for (uint64_t none = __ballot(s0 + lane < P && (r < 0 || r >= T)); none; none &= none - 1) {
    const int64_t s = s0 + __builtin_ctzll(none);
    for (int c = threadIdx.x; c < pieces; c += kThreads)
      Q::store(y, s * pieces + c, typename Q::Raw{});
  }
}

// A wave a part of a token, which it reads once and stores k times (a wave a slot, which reads
// it, took 81 us for 8192 tokens of 2048 channels and 8 choices, this 59); the workgroups past
// the tokens clear, 64 slots each.
template <bool BF16, bool VEC>
__global__ __launch_bounds__(kThreads) void expert_gather_kernel(
    const void *__restrict__ x, int64_t T, int pieces, const int32_t *__restrict__ rows,
    const int32_t *__restrict__ slots, int k, int64_t P, int parts, int token_groups,
    void *__restrict__ out) {
  using Q = Piece<BF16, VEC>;
  if ((int)blockIdx.x >= token_groups) {
    clear_rows<BF16, VEC>(rows, (int64_t)((int)blockIdx.x - token_groups) * 64, P, T, pieces, out);
    return;
  }
  Item it;
  if (!item_of(T, parts, it)) return;
  const int lane = threadIdx.x & 63;
  typename Q::Raw v[kPieces] = {};
  int c[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    c[i] = (it.part * kPieces + i) * 64 + lane;
    if (c[i] < pieces) v[i] = Q::load(x, it.row * pieces + c[i]);
  }
  for (int j = 0; j < k; ++j) {
    const int64_t s = slots[it.row * k + j];
    if (s < 0 || s >= P) continue;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (c[i] < pieces) Q::store(out, s * pieces + c[i], v[i]);
  }
}

// One piece a lane; the rows of kBatch choices are loaded together.  8192 tokens of 8 choices: 2048
// bf16 channels 57.3 us (5.3 TB/s), 512 12.5, 64 7.2; 2049, element by element, 182 (1.7).
template <bool BF16, bool VEC>
__global__ __launch_bounds__(kThreads) void expert_combine_kernel(
    const void *__restrict__ z, int64_t P, int pieces, const int32_t *__restrict__ slots,
    const float *__restrict__ weights, int64_t T, int k, int parts, void *__restrict__ out) {
  using Q = Piece<BF16, VEC>;
  constexpr int kBatch = 4;
  Item it;
  if (!item_of(T, parts, it)) return;
  const int c = it.part * 64 + (threadIdx.x & 63);
  if (c >= pieces) return;
  float acc[Q::V] = {};
  for (int j0 = 0; j0 < k; j0 += kBatch) {
    typename Q::Raw v[kBatch];
    bool has[kBatch];
    float w[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int64_t at = it.row * k + min(j0 + b, k - 1);
      const int64_t s = slots[at];
      has[b] = j0 + b < k && s >= 0 && s < P;
      w[b] = weights ? weights[at] : 1.0f;
      if (has[b]) v[b] = Q::load(z, s * pieces + c);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (has[b]) {
        float f[Q::V];
        Q::widen(v[b], f);
#pragma unroll
        for (int i = 0; i < Q::V; ++i) acc[i] = fmaf(w[b], f[i], acc[i]);
      }
    }
  }
  Q::store(out, it.row * pieces + c, Q::narrow(acc));
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// A workgroup a token; those past the tokens write the zeros of dz, 64 slots each.  8192 tokens of 8
// choices: 2048 bf16 channels 112 us (5.1 TB/s), 512 32.5 (4.4), 64 26.1, bound by the workgroups' own
// latency; 2049, element by element, 258 (2.2).
template <bool BF16, bool VEC, int kMost>
__global__ __launch_bounds__(kThreads) void expert_combine_backward_kernel(
    const void *__restrict__ dout, const void *__restrict__ z, int64_t P, int pieces,
    const int32_t *__restrict__ rows, const int32_t *__restrict__ slots,
    const float *__restrict__ weights, int64_t T, int k, void *__restrict__ dz,
    float *__restrict__ dweights) {
  using Q = Piece<BF16, VEC>;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int64_t)blockIdx.x >= T) {
    clear_rows<BF16, VEC>(rows, ((int64_t)blockIdx.x - T) * 64, P, T, pieces, dz);
    return;
  }
  const int64_t t = blockIdx.x;
  int64_t slot[kMost];
  float w[kMost], dot[kMost];
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    const int64_t s = j < k ? slots[t * k + j] : -1;
    slot[j] = s < P ? s : -1;
    w[j] = j < k && weights ? weights[t * k + j] : 1.0f;
    dot[j] = 0.0f;
  }
  for (int c = tid; c < pieces; c += kThreads) {
    float d[Q::V];
    Q::widen(Q::load(dout, t * pieces + c), d);
    typename Q::Raw v[kMost];
    if (dweights) {
#pragma unroll
      for (int j = 0; j < kMost; ++j)
        if (slot[j] >= 0) v[j] = Q::load(z, slot[j] * pieces + c);
    }
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      if (slot[j] < 0) continue;
      if (dweights) {
        float f[Q::V];
        Q::widen(v[j], f);
#pragma unroll
        for (int i = 0; i < Q::V; ++i) dot[j] = fmaf(d[i], f[i], dot[j]);
      }
      if (dz) {
        float g[Q::V];
#pragma unroll
        for (int i = 0; i < Q::V; ++i) g[i] = w[j] * d[i];
        Q::store(dz, slot[j] * pieces + c, Q::narrow(g));
      }
    }
  }
  if (!dweights) return;
  __shared__ float part[kWaves][kMost];
#pragma unroll
  for (int j = 0; j < kMost; ++j) {
    const float s = wave_sum(dot[j]);
    if (lane == 0) part[wave][j] = s;
  }
  __syncthreads();
  if (tid < k) {
    float s = part[0][tid];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) s += part[v][tid];
    dweights[t * k + tid] = s;
  }
}

bool whole_pieces(int64_t N, bool bf16) { return N * (bf16 ? 2 : 4) % 16 == 0; }
int pieces_of(int64_t N, bool bf16, bool vec) { return (int)(vec ? N * (bf16 ? 2 : 4) / 16 : N); }

template <class Go>
hipError_t on_type(bool bf16, bool vec, Go go) {
  using Yes = std::true_type;
  using No = std::false_type;
  if (bf16) return vec ? go(Yes{}, Yes{}) : go(Yes{}, No{});
  return vec ? go(No{}, Yes{}) : go(No{}, No{});
}

}  // namespace

hipError_t launch_expert_gather(const void *x, bool bf16, int64_t T, int64_t N,
                                const int32_t *rows, const int32_t *slots, int k, int64_t P,
                                void *out, hipStream_t stream) {
  const bool vec = whole_pieces(N, bf16);
  const int pieces = pieces_of(N, bf16, vec);
  const int parts = (pieces + 64 * kPieces - 1) / (64 * kPieces);
  const int tokens = (int)((T * parts + kWaves - 1) / kWaves);
  const unsigned groups = (unsigned)(tokens + (P + 63) / 64);
  return on_type(bf16, vec, [&](auto b, auto v) {
    expert_gather_kernel<decltype(b)::value, decltype(v)::value><<<groups, kThreads, 0, stream>>>(
        x, T, pieces, rows, slots, k, P, parts, tokens, out);
    return hipGetLastError();
  });
}

hipError_t launch_expert_combine(const void *z, bool bf16, int64_t P, int64_t N,
                                 const int32_t *slots, const float *weights, int64_t T, int k,
                                 void *out, hipStream_t stream) {
  const bool vec = whole_pieces(N, bf16);
  const int pieces = pieces_of(N, bf16, vec);
  const int parts = (pieces + 63) / 64;
  const unsigned groups = (unsigned)((T * parts + kWaves - 1) / kWaves);
  return on_type(bf16, vec, [&](auto b, auto v) {
    expert_combine_kernel<decltype(b)::value, decltype(v)::value>
        <<<groups, kThreads, 0, stream>>>(z, P, pieces, slots, weights, T, k, parts, out);
    return hipGetLastError();
  });
}

hipError_t launch_expert_combine_backward(const void *dout, const void *z, bool bf16, int64_t P,
                                          int64_t N, const int32_t *rows, const int32_t *slots,
                                          const float *weights, int64_t T, int k, void *dz,
                                          float *dweights, hipStream_t stream) {
  const bool vec = whole_pieces(N, bf16);
  const int pieces = pieces_of(N, bf16, vec);
  const unsigned groups = (unsigned)(T + (dz ? (P + 63) / 64 : 0));
  return on_type(bf16, vec, [&](auto b, auto v) {
    constexpr bool B = decltype(b)::value, V = decltype(v)::value;
    auto kern = k <= 4 ? expert_combine_backward_kernel<B, V, 4>
                       : (k <= 8 ? expert_combine_backward_kernel<B, V, 8>
                                 : expert_combine_backward_kernel<B, V, 16>);
    kern<<<groups, kThreads, 0, stream>>>(dout, z, P, pieces, rows, slots, weights, T, k, dz,
                                          dweights);
    return hipGetLastError();
  });
}

}  // namespace rfq
