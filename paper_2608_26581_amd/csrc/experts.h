// Internal declarations of the calls around a layer of experts (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rfq.h"

namespace rfq {

// Confirms that the current device is a gfx950 GPU (cached per device).
rfq_status check_device();

// Experts of a router or a product, and choices of a token, at most.
constexpr int64_t kMaxExperts = 1024;
constexpr int64_t kMaxChoices = 16;

hipError_t launch_route(const void *logits, bool bf16, int64_t T, int E, int k, bool renormalize,
                        float *weights, int32_t *experts, hipStream_t stream);
hipError_t launch_route_backward(const float *dweights, const void *logits, bool bf16, int64_t T,
                                 int E, int k, const float *weights, const int32_t *experts,
                                 bool renormalize, void *dlogits, hipStream_t stream);

// Workspace of the sort (0: one workgroup sorts); with less, one workgroup sorts.
int64_t expert_sort_workspace(int64_t T, int64_t k, int64_t E);
hipError_t launch_expert_sort(const int32_t *experts, int64_t T, int k, int64_t first, int E,
                              int32_t *offsets, int32_t *rows, int32_t *slots, void *workspace,
                              int64_t workspace_bytes, hipStream_t stream);

hipError_t launch_expert_gather(const void *x, bool bf16, int64_t T, int64_t N,
                                const int32_t *rows, const int32_t *slots, int k, int64_t P,
                                void *out, hipStream_t stream);
// weights == nullptr: ones.
hipError_t launch_expert_combine(const void *z, bool bf16, int64_t P, int64_t N,
                                 const int32_t *slots, const float *weights, int64_t T, int k,
                                 void *out, hipStream_t stream);
// dz or dweights may be nullptr.
hipError_t launch_expert_combine_backward(const void *dout, const void *z, bool bf16, int64_t P,
                                          int64_t N, const int32_t *rows, const int32_t *slots,
                                          const float *weights, int64_t T, int k, void *dz,
                                          float *dweights, hipStream_t stream);

struct ExpertsGemm {
  const uint8_t *qc, *qs, *rc, *rs;   // activations [M] (rc == nullptr: primary only)
  const uint8_t *wc, *ws;             // weights [E][N]
  const int32_t *offsets;             // [E + 1]
  const int32_t *rows;                // [P], or nullptr: row p is slot p's
  int64_t M, P, N, K;                 // M > 0
  int E;
  void *z;                            // [P][N]
};
// Whether the tiles of the product can be numbered.
bool gemm_experts_fits(int64_t P, int64_t E, int64_t N);
hipError_t launch_gemm_experts(const ExpertsGemm &g, bool z_bf16, hipStream_t stream);

}  // namespace rfq
