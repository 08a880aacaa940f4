// C ABI of the key/value cache calls: host-side argument validation and dispatch,
// in the order of the other calls (dtype, shape, empty work, pointers, alignment,
// device).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv.h"
#include "rfq.h"

namespace {

using rfq::check_device;

constexpr int64_t kMaxWorkItems = UINT32_MAX;
constexpr int64_t kMaxHeads = 1 << 16;
// Strides (elements) and sizes below keep every address within 63 bits.
constexpr int64_t kMaxStride = int64_t(1) << 40;

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool valid_dtype(rfq_dtype d) { return d == RFQ_F32 || d == RFQ_BF16; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
rfq_status launched(hipError_t e) { return e == hipSuccess ? RFQ_OK : RFQ_ERR_LAUNCH; }

bool page_ok(int64_t page) { return page >= 16 && page <= 256 && (page & (page - 1)) == 0; }

bool strides_ok(const rfq_heads &h, bool output, int64_t T, int64_t H) {
  const int64_t low = output ? 1 : 0;
  return (T <= 1 || h.token_stride >= low) && (H <= 1 || h.head_stride >= low) &&
         h.token_stride >= 0 && h.head_stride >= 0 && h.token_stride <= kMaxStride &&
         h.head_stride <= kMaxStride;
}
bool heads_aligned(const rfq_heads &h, int64_t bytes) {
  return aligned(h.data, 16) && h.token_stride * bytes % 16 == 0 && h.head_stride * bytes % 16 == 0;
}

rfq_status check_rope(const rfq_rope_spec &r, int64_t D) {
  if (r.rotary < 16 || r.rotary % 16 != 0 || r.rotary > D || r.n_axes < 1 ||
      r.n_axes > rfq::kMaxAxes || r.max_pos < 0 || r.positions_stride < 0 ||
      r.positions_stride > kMaxStride)
    return RFQ_ERR_SHAPE;
  if (r.axes)
    for (int j = 0; j < r.rotary / 2; ++j)
      if (r.axes[j] >= r.n_axes) return RFQ_ERR_SHAPE;
  return RFQ_OK;
}
rfq_status check_rope_pointers(const rfq_rope_spec &r) {
  if (!r.positions || (!r.cos_sin && r.max_pos > 0)) return RFQ_ERR_NULL;
  if (!aligned(r.positions, 4) || !aligned(r.cos_sin, 8)) return RFQ_ERR_ALIGN;
  return RFQ_OK;
}

rfq_status check_cache(const rfq_kv_cache &c) {
  if ((c.D != 64 && c.D != 128 && c.D != 256) || !page_ok(c.page) || c.heads < 1 ||
      c.heads > kMaxHeads || c.blocks < 0 || c.blocks > INT32_MAX / c.page)
    return RFQ_ERR_SHAPE;
  return RFQ_OK;
}
rfq_status check_cache_pointers(const rfq_kv_cache &c) {
  if (!c.k_codes || !c.k_scales || !c.v_codes || !c.v_scales) return RFQ_ERR_NULL;
  if (!aligned(c.k_codes, 16) || !aligned(c.k_scales, 16) || !aligned(c.v_codes, 16) ||
      !aligned(c.v_scales, 16))
    return RFQ_ERR_ALIGN;
  return RFQ_OK;
}

rfq_status rope_call(const rfq_heads *x, rfq_dtype dtype, int64_t T, int64_t H, int64_t D,
                     const rfq_rope_spec *rope, const rfq_heads *y, bool backward,
                     void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (!x || !y || !rope) return RFQ_ERR_NULL;
  if (T < 0 || H < 0 || D < 16 || D % 16 != 0 || D > rfq::kMaxHeadDim || H > kMaxHeads ||
      T > kMaxWorkItems / 256 || !strides_ok(*x, false, T, H) || !strides_ok(*y, true, T, H))
    return RFQ_ERR_SHAPE;
  rfq_status s = check_rope(*rope, D);
  if (s != RFQ_OK) return s;
  if (T == 0 || H == 0) return RFQ_OK;
  if (!x->data || !y->data) return RFQ_ERR_NULL;
  if ((s = check_rope_pointers(*rope)) != RFQ_OK) return s;
  const int64_t bytes = dtype == RFQ_BF16 ? 2 : 4;
  if (!heads_aligned(*x, bytes) || !heads_aligned(*y, bytes)) return RFQ_ERR_ALIGN;
  if ((s = check_device()) != RFQ_OK) return s;
  return launched(rfq::launch_rope(*x, dtype == RFQ_BF16, T, H, D, *rope, backward, *y,
                                   static_cast<hipStream_t>(hip_stream)));
}

// A workspace query takes the sizes that the call takes.  One head and request can have all
// T * Hq rows, in tiles of up to kWideRows: the last tile's end is a 32-bit number too.
bool attention_sizes_ok(int64_t T, int64_t Hq, int64_t heads, int64_t B) {
  constexpr int64_t most = int64_t(1) << 24, rows = INT32_MAX - (rfq::kWideRows - 1);
  return T >= 0 && T < most && B >= 0 && B < most && heads >= 1 && heads <= kMaxHeads &&
         Hq >= heads && Hq <= kMaxHeads && Hq % heads == 0 && T * Hq <= rows;
}

}  // namespace

extern "C" {

rfq_status rfq_block_assign(const int32_t *ctx_lens, const int32_t *new_lens, int64_t B,
                            int32_t *block_tables, int64_t width, const int32_t *free_blocks,
                            int64_t n_free, const int32_t *free_count, int64_t page,
                            int64_t tokens, int32_t *slots, int32_t *positions,
                            int32_t *seq_lens, int32_t *query_starts, int32_t *counts,
                            void *hip_stream) {
  if (B < 0 || B > rfq::kMaxBlockRequests || width < 0 || width > INT32_MAX || n_free < 0 ||
      n_free > INT32_MAX || tokens < 0 || tokens > INT32_MAX || !page_ok(page))
    return RFQ_ERR_SHAPE;
  if (!free_count || !query_starts || !counts || (n_free > 0 && !free_blocks) ||
      (B > 0 && (!ctx_lens || !new_lens || !seq_lens || (width > 0 && !block_tables))) ||
      (tokens > 0 && (!slots || !positions)))
    return RFQ_ERR_NULL;
  for (const void *p : {(const void *)ctx_lens, (const void *)new_lens, (const void *)block_tables,
                        (const void *)free_blocks, (const void *)free_count, (const void *)slots,
                        (const void *)positions, (const void *)seq_lens,
                        (const void *)query_starts, (const void *)counts})
    if (!aligned(p, 4)) return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_block_assign(ctx_lens, new_lens, (int)B, block_tables, width,
                                           free_blocks, n_free, free_count, (int)page, tokens,
                                           slots, positions, seq_lens, query_starts, counts,
                                           static_cast<hipStream_t>(hip_stream)));
}

rfq_status rfq_block_release(const int32_t *lens, const uint8_t *ended, int64_t B,
                             const int32_t *block_tables, int64_t width, int32_t *free_blocks,
                             int64_t n_free, const int32_t *free_count, int64_t page,
                             int32_t *free_count_out, void *hip_stream) {
  if (B < 0 || B > rfq::kMaxBlockRequests || width < 0 || width > INT32_MAX || n_free < 0 ||
      n_free > INT32_MAX || !page_ok(page))
    return RFQ_ERR_SHAPE;
  if (!free_count || !free_count_out || (n_free > 0 && !free_blocks) ||
      (B > 0 && (!lens || !ended || (width > 0 && !block_tables))))
    return RFQ_ERR_NULL;
  for (const void *p : {(const void *)lens, (const void *)block_tables, (const void *)free_blocks,
                        (const void *)free_count, (const void *)free_count_out})
    if (!aligned(p, 4)) return RFQ_ERR_ALIGN;
  const rfq_status s = check_device();
  if (s != RFQ_OK) return s;
  return launched(rfq::launch_block_release(lens, ended, (int)B, block_tables, width, free_blocks,
                                            n_free, free_count, (int)page, free_count_out,
                                            static_cast<hipStream_t>(hip_stream)));
}

rfq_status rfq_rope(const rfq_heads *x, rfq_dtype dtype, int64_t T, int64_t H, int64_t D,
                    const rfq_rope_spec *rope, const rfq_heads *y, void *hip_stream) {
  return rope_call(x, dtype, T, H, D, rope, y, false, hip_stream);
}

rfq_status rfq_rope_backward(const rfq_heads *dy, rfq_dtype dtype, int64_t T, int64_t H,
                             int64_t D, const rfq_rope_spec *rope, const rfq_heads *dx,
                             void *hip_stream) {
  return rope_call(dy, dtype, T, H, D, rope, dx, true, hip_stream);
}

rfq_status rfq_kv_append(const rfq_heads *k, const rfq_heads *v, rfq_dtype dtype, int64_t T,
                         const int32_t *slots, const rfq_kv_cache *cache, const rfq_heads *q,
                         int64_t Hq, const rfq_rope_spec *rope, const rfq_heads *q_out,
                         void *hip_stream) {
  if (!valid_dtype(dtype)) return RFQ_ERR_DTYPE;
  if (!k || !v || !cache || (q == nullptr) != (q_out == nullptr) || (q && !rope))
    return RFQ_ERR_NULL;
  rfq_status s = check_cache(*cache);
  if (s != RFQ_OK) return s;
  const int64_t D = cache->D, heads = cache->heads;
  if (T < 0 || Hq < 0 || Hq > kMaxHeads || !strides_ok(*k, false, T, heads) ||
      !strides_ok(*v, false, T, heads) ||
      (q && (!strides_ok(*q, false, T, Hq) || !strides_ok(*q_out, true, T, Hq))))
    return RFQ_ERR_SHAPE;
  if (rope && (s = check_rope(*rope, D)) != RFQ_OK) return s;
  // One workgroup per token and 256 work items of it.
  const int64_t items = (q ? up(Hq * (D / 16), 64) * 64 : 0) + 2 * (up(heads * (D / 8), 64) * 64);
  if (T > kMaxWorkItems / (up(items, 256) * 256)) return RFQ_ERR_SHAPE;
  if (T == 0) return RFQ_OK;
  if (!k->data || !v->data || !slots || (q && Hq > 0 && (!q->data || !q_out->data)))
    return RFQ_ERR_NULL;
  if ((s = check_cache_pointers(*cache)) != RFQ_OK) return s;
  if (rope && (s = check_rope_pointers(*rope)) != RFQ_OK) return s;
  const int64_t bytes = dtype == RFQ_BF16 ? 2 : 4;
  if (!heads_aligned(*k, bytes) || !heads_aligned(*v, bytes) || !aligned(slots, 4) ||
      (q && (!heads_aligned(*q, bytes) || !heads_aligned(*q_out, bytes))))
    return RFQ_ERR_ALIGN;
  if ((s = check_device()) != RFQ_OK) return s;
  return launched(rfq::launch_kv_append(*k, *v, dtype == RFQ_BF16, T, slots, *cache, q, Hq, rope,
                                        q_out, static_cast<hipStream_t>(hip_stream)));
}

rfq_status rfq_kv_gather(const rfq_kv_cache *cache, const int32_t *slots, int64_t n,
                         void *k_out, void *v_out, rfq_dtype out_dtype, void *hip_stream) {
  if (!valid_dtype(out_dtype)) return RFQ_ERR_DTYPE;
  if (!cache) return RFQ_ERR_NULL;
  rfq_status s = check_cache(*cache);
  if (s != RFQ_OK) return s;
  if (n < 0 || n > kMaxWorkItems / (up(2 * cache->heads * (cache->D / 8), 256) * 256))
    return RFQ_ERR_SHAPE;
  if (n == 0) return RFQ_OK;
  if (!slots || !k_out || !v_out) return RFQ_ERR_NULL;
  if ((s = check_cache_pointers(*cache)) != RFQ_OK) return s;
  if (!aligned(slots, 4) || !aligned(k_out, 16) || !aligned(v_out, 16)) return RFQ_ERR_ALIGN;
  if ((s = check_device()) != RFQ_OK) return s;
  return launched(rfq::launch_kv_gather(*cache, slots, n, k_out, v_out, out_dtype == RFQ_BF16,
                                        static_cast<hipStream_t>(hip_stream)));
}

int64_t rfq_kv_attention_workspace_bytes(int64_t T, int64_t Hq, int64_t heads, int64_t D,
                                         int64_t B, int64_t max_query, int64_t max_seq) {
  if (!attention_sizes_ok(T, Hq, heads, B) || (D != 64 && D != 128 && D != 256) ||
      max_query < 0 || max_query > INT32_MAX || max_seq < 0 || T == 0 || B == 0)
    return 0;
  return rfq::kv_attention_workspace(T, Hq, heads, D, B, max_query, max_seq);
}

rfq_status rfq_kv_attention(const rfq_heads *q, int64_t T, int64_t Hq, const rfq_kv_cache *cache,
                            const int32_t *block_tables, int64_t width,
                            const int32_t *seq_lens, const int32_t *query_starts, int64_t B,
                            int64_t max_query, int64_t max_seq, float scale, int causal,
                            int64_t window, const rfq_heads *out, float *lse,
                            void *workspace, int64_t workspace_bytes, void *hip_stream) {
  if (!q || !cache || !out) return RFQ_ERR_NULL;
  rfq_status s = check_cache(*cache);
  if (s != RFQ_OK) return s;
  if (!attention_sizes_ok(T, Hq, cache->heads, B) || width < 0 || width > INT32_MAX ||
      max_query < 0 || max_query > INT32_MAX || max_seq < 0 || window < 0 ||
      workspace_bytes < 0 || !strides_ok(*q, false, T, Hq) || !strides_ok(*out, true, T, Hq))
    return RFQ_ERR_SHAPE;
  if (T == 0 || B == 0) return RFQ_OK;
  if (cache->blocks == 0) return RFQ_ERR_SHAPE;
  if (!q->data || !out->data || !seq_lens || !query_starts || (width > 0 && !block_tables) ||
      (!workspace && workspace_bytes > 0))
    return RFQ_ERR_NULL;
  if ((s = check_cache_pointers(*cache)) != RFQ_OK) return s;
  if (!heads_aligned(*q, 2) || !heads_aligned(*out, 2) || !aligned(block_tables, 4) ||
      !aligned(seq_lens, 4) || !aligned(query_starts, 4) || !aligned(lse, 4) ||
      !aligned(workspace, 16))
    return RFQ_ERR_ALIGN;
  if ((s = check_device()) != RFQ_OK) return s;
  rfq::AttentionArgs a = {};
  a.q = static_cast<const uint16_t *>(q->data);
  a.q_ts = q->token_stride;
  a.q_hs = q->head_stride;
  a.k_codes = cache->k_codes;
  a.k_scales = cache->k_scales;
  a.v_codes = cache->v_codes;
  a.v_scales = cache->v_scales;
  a.tables = block_tables;
  a.lens = seq_lens;
  a.starts = query_starts;
  a.width = width;
  a.T = (int32_t)T;
  a.Hq = (int32_t)Hq;
  a.heads = (int32_t)cache->heads;
  a.group = (int32_t)(Hq / cache->heads);
  a.blocks = (int32_t)cache->blocks;
  a.page = (int32_t)cache->page;
  a.page_shift = __builtin_ctz((unsigned)cache->page);
  a.B = (int32_t)B;
  // Token numbers stay well inside 32 bits (tiles are counted past the end).
  constexpr int64_t kMostTokens = int64_t(1) << 30;
  const int64_t tokens = width > kMostTokens / cache->page ? kMostTokens : width * cache->page;
  a.capacity = (int32_t)tokens;
  a.causal = causal != 0;
  a.window = (int32_t)(window > kMostTokens ? 0 : window);   // wider than any request: none
  a.scale_log2 = scale * 1.4426950408889634f;
  a.out = static_cast<uint16_t *>(out->data);
  a.o_ts = out->token_stride;
  a.o_hs = out->head_stride;
  a.lse = lse;
  return launched(rfq::launch_kv_attention(a, cache->D, max_query, max_seq,
                                           static_cast<float *>(workspace), workspace_bytes,
                                           static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
