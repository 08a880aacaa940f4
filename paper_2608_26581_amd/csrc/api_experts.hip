// C ABI of the calls around a layer of experts: host-side argument validation and
// dispatch, in the order of the other calls (dtype, shape, empty work, pointers, alignment,
// device).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts.h"
#include "rfq.h"

namespace {

using rfq::check_device;

constexpr int64_t kMaxWorkItems = UINT32_MAX;

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool valid_dtype(rfq_dtype d) { return d == RFQ_F32 || d == RFQ_BF16; }
int64_t size_of(rfq_dtype d) { return d == RFQ_BF16 ? 2 : 4; }
rfq_status launched(hipError_t e) { return e == hipSuccess ? RFQ_OK : RFQ_ERR_LAUNCH; }
hipStream_t stream_of(void *s) { return static_cast<hipStream_t>(s); }

// T tokens with k choices: pairs are numbered in 32 bits.
bool pairs_ok(int64_t T, int64_t k) {
  return T >= 0 && k >= 1 && k <= rfq::kMaxChoices && T <= INT32_MAX / k;
}
// A router's sizes: the launch covers 4 rows a wave, or one.
bool route_ok(int64_t T, int64_t E, int64_t k) {
  return pairs_ok(T, k) && E >= k && E <= rfq::kMaxExperts && T <= kMaxWorkItems / 64 - 4;
}
// Rows of N elements that waves go through in parts of 64 pieces (of 16 bytes, or of an
// element), and with them workgroups of 256 for 64 of P slots.
int64_t row_parts(int64_t rows, int64_t N, rfq_dtype dtype) {
  const int64_t bytes = N * size_of(dtype);
  const int64_t pieces = bytes % 16 == 0 ? bytes / 16 : N;
  return rows * ((pieces + 63) / 64);
}
bool rows_ok(int64_t rows, int64_t N, rfq_dtype dtype, int64_t P = 0) {
  // (A lane's piece numbers go up to 256 past the row's last, in 32 bits.)
  if (rows < 0 || rows > INT32_MAX || N < 0 || N >= INT32_MAX - 255) return false;
  return row_parts(rows, N, dtype) + 4 * (P / 64) <= kMaxWorkItems / 64 - 16;
}

}  // namespace

extern "C" {

rfq_status rfq_route(const void *logits, rfq_dtype dtype, int64_t T, int64_t E, int64_t k,
                     int renormalize, float *weights, int32_t *experts, void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (!route_ok(T, E, k)) return RFQ_ERR_SHAPE;
  if (T == 0) return RFQ_OK;
  if (!logits || !weights || !experts) return RFQ_ERR_NULL;
  if (!aligned(logits, size_of(dtype)) || !aligned(weights, 4) || !aligned(experts, 4))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_route(logits, dtype == RFQ_BF16, T, (int)E, (int)k, renormalize != 0,
                                    weights, experts, stream_of(hip_stream)));
}

rfq_status rfq_route_backward(const float *dweights, const void *logits, rfq_dtype dtype,
                              int64_t T, int64_t E, int64_t k, const float *weights,
                              const int32_t *experts, int renormalize, void *dlogits,
                              void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (!route_ok(T, E, k)) return RFQ_ERR_SHAPE;
  if (T == 0) return RFQ_OK;
  if (!dweights || !logits || !weights || !experts || !dlogits) return RFQ_ERR_NULL;
  if (!aligned(logits, size_of(dtype)) || !aligned(dlogits, size_of(dtype)) ||
      !aligned(dweights, 4) || !aligned(weights, 4) || !aligned(experts, 4))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_route_backward(dweights, logits, dtype == RFQ_BF16, T, (int)E, (int)k,
                                             weights, experts, renormalize != 0, dlogits,
                                             stream_of(hip_stream)));
}

int64_t rfq_expert_sort_workspace_bytes(int64_t T, int64_t k, int64_t E) {
  if (!pairs_ok(T, k) || E < 1 || E > rfq::kMaxExperts) return 0;
  return rfq::expert_sort_workspace(T, k, E);
}

rfq_status rfq_expert_sort(const int32_t *experts, int64_t T, int64_t k, int64_t first, int64_t E,
                           int32_t *offsets, int32_t *rows, int32_t *slots, void *workspace,
                           int64_t workspace_bytes, void *hip_stream) {
  if (!pairs_ok(T, k) || E < 1 || E > rfq::kMaxExperts || first < INT32_MIN || first > INT32_MAX ||
      workspace_bytes < 0)
    return RFQ_ERR_SHAPE;
  if (!offsets || (T > 0 && (!experts || !rows || !slots)) || (!workspace && workspace_bytes > 0))
    return RFQ_ERR_NULL;
  if (!aligned(experts, 4) || !aligned(offsets, 4) || !aligned(rows, 4) || !aligned(slots, 4) ||
      !aligned(workspace, 16))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_expert_sort(experts, T, (int)k, first, (int)E, offsets, rows, slots,
                                          workspace, workspace_bytes, stream_of(hip_stream)));
}

rfq_status rfq_expert_gather(const void *x, rfq_dtype dtype, int64_t T, int64_t N,
                             const int32_t *rows, const int32_t *slots, int64_t k, int64_t P,
                             void *out, void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (P < 0 || P > INT32_MAX || !pairs_ok(T, k) || !rows_ok(T, N, dtype, P))
    return RFQ_ERR_SHAPE;
  if (P == 0 || N == 0) return RFQ_OK;
  if ((T > 0 && (!x || !slots)) || !rows || !out) return RFQ_ERR_NULL;
  if (!aligned(x, 16) || !aligned(rows, 4) || !aligned(slots, 4) || !aligned(out, 16))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_expert_gather(x, dtype == RFQ_BF16, T, N, rows, slots, (int)k, P, out,
                                            stream_of(hip_stream)));
}

rfq_status rfq_expert_combine(const void *z, rfq_dtype dtype, int64_t P, int64_t N,
                              const int32_t *slots, const float *weights, int64_t T, int64_t k,
                              void *out, void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (P < 0 || P > INT32_MAX || !pairs_ok(T, k) || !rows_ok(T, N, dtype)) return RFQ_ERR_SHAPE;
  if (T == 0 || N == 0) return RFQ_OK;
  if ((P > 0 && !z) || !slots || !out) return RFQ_ERR_NULL;
  if (!aligned(z, 16) || !aligned(slots, 4) || !aligned(weights, 4) || !aligned(out, 16))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_expert_combine(z, dtype == RFQ_BF16, P, N, slots, weights, T, (int)k,
                                             out, stream_of(hip_stream)));
}

rfq_status rfq_expert_combine_backward(const void *dout, const void *z, rfq_dtype dtype, int64_t P,
                                       int64_t N, const int32_t *rows, const int32_t *slots,
                                       const float *weights, int64_t T, int64_t k, void *dz,
                                       float *dweights, void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  // A workgroup of 256 a token, and one for 64 slots.
  if (P < 0 || P > INT32_MAX || !pairs_ok(T, k) || !rows_ok(T, N, dtype) ||
      T + P / 64 + 1 > kMaxWorkItems / 256)
    return RFQ_ERR_SHAPE;
  if ((!dz || P == 0 || N == 0) && (!dweights || T == 0)) return RFQ_OK;
  if ((T > 0 && N > 0 && !dout) || (T > 0 && !slots) || (P > 0 && dz && !rows) ||
      (P > 0 && N > 0 && dweights && !z))
    return RFQ_ERR_NULL;
  if (!aligned(dout, 16) || !aligned(z, 16) || !aligned(rows, 4) || !aligned(slots, 4) ||
      !aligned(weights, 4) || !aligned(dz, 16) || !aligned(dweights, 4))
    return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_expert_combine_backward(dout, z, dtype == RFQ_BF16, P, N, rows, slots,
                                                      weights, T, (int)k, dz, dweights,
                                                      stream_of(hip_stream)));
}

rfq_status rfq_gemm_experts(const uint8_t *q_codes, const uint8_t *q_scales,
                            const uint8_t *r_codes, const uint8_t *r_scales,
                            const uint8_t *w_codes, const uint8_t *w_scales,
                            const int32_t *offsets, const int32_t *rows, int64_t M, int64_t P,
                            int64_t E, int64_t N, int64_t K, void *z, rfq_dtype z_dtype,
                            void *hip_stream) {
  if (!valid_dtype(z_dtype)) return RFQ_ERR_DTYPE;
  constexpr int64_t most = int64_t(1) << 31;
  if (M < 0 || P < 0 || E < 0 || N < 0 || K < 32 || K % 32 != 0 || K > most || M >= most ||
      P >= most - 256 || E > rfq::kMaxExperts || N >= most - 256 || (!rows && P != M) ||
      M * (K / 2) >= most || N * (K / 2) >= most || !rfq::gemm_experts_fits(P, E, N))
    return RFQ_ERR_SHAPE;
  if (P == 0 || N == 0 || E == 0) return RFQ_OK;
  if (M == 0) return RFQ_ERR_SHAPE;
  if (!q_codes || !q_scales || !w_codes || !w_scales || !offsets || !z) return RFQ_ERR_NULL;
  if ((r_codes == nullptr) != (r_scales == nullptr)) return RFQ_ERR_NULL;
  for (const void *p : {(const void *)q_codes, (const void *)q_scales, (const void *)r_codes,
                        (const void *)r_scales, (const void *)w_codes, (const void *)w_scales,
                        (const void *)z})
    if (!aligned(p, 16)) return RFQ_ERR_ALIGN;
  if (!aligned(offsets, 4) || !aligned(rows, 4)) return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  const rfq::ExpertsGemm g{q_codes, q_scales, r_codes, r_scales, w_codes, w_scales, offsets, rows,
                           M, P, N, K, (int)E, z};
  return launched(rfq::launch_gemm_experts(g, z_dtype == RFQ_BF16, stream_of(hip_stream)));
}

}  // extern "C"
