// Internal declarations of the key/value cache calls (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rfq.h"

namespace rfq {

// Confirms that the current device is a gfx950 GPU (cached per device).
rfq_status check_device();

// Requests of one call to the block calls: two int32 per request in LDS.
constexpr int64_t kMaxBlockRequests = 16384;
// Channels of a head, at most, and position axes.
constexpr int kMaxHeadDim = 512;
constexpr int kMaxAxes = 8;

hipError_t launch_block_assign(const int32_t *ctx, const int32_t *fresh, int B, int32_t *tables,
                               int64_t width, const int32_t *free_blocks, int64_t n_free,
                               const int32_t *free_count, int page, int64_t tokens,
                               int32_t *slots, int32_t *positions, int32_t *seq_lens,
                               int32_t *query_starts, int32_t *counts, hipStream_t stream);
hipError_t launch_block_release(const int32_t *lens, const uint8_t *ended, int B,
                                const int32_t *tables, int64_t width, int32_t *free_blocks,
                                int64_t n_free, const int32_t *free_count, int page,
                                int32_t *count_out, hipStream_t stream);

// y = rotation of x [T][H][D] (backward: by the opposite angle); checked arguments.
hipError_t launch_rope(const rfq_heads &x, bool bf16, int64_t T, int64_t H, int64_t D,
                       const rfq_rope_spec &rope, bool backward, const rfq_heads &y,
                       hipStream_t stream);
// rope == nullptr: k is not rotated and there is no q.
hipError_t launch_kv_append(const rfq_heads &k, const rfq_heads &v, bool bf16, int64_t T,
                            const int32_t *slots, const rfq_kv_cache &cache, const rfq_heads *q,
                            int64_t Hq, const rfq_rope_spec *rope, const rfq_heads *q_out,
                            hipStream_t stream);
hipError_t launch_kv_gather(const rfq_kv_cache &cache, const int32_t *slots, int64_t n,
                            void *k_out, void *v_out, bool bf16, hipStream_t stream);

struct AttentionArgs {
  const uint16_t *q;
  int64_t q_ts, q_hs;
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  const int32_t *tables, *lens, *starts;
  int64_t width;
  int32_t T, Hq, heads, group, blocks, page, page_shift, B;
  int32_t capacity;                 // tokens a table row can name
  int32_t most_rows;                // requests with more are another launch's
  int32_t causal;
  int32_t window;                   // 0: none
  float scale_log2;                 // scale * log2(e)
  uint16_t *out;
  int64_t o_ts, o_hs;
  float *lse;
};
int64_t kv_attention_workspace(int64_t T, int64_t Hq, int64_t heads, int64_t D, int64_t B,
                               int64_t max_query, int64_t max_seq);
// The wide kernel: requests with more than few_rows rows (queries times group), in row
// tiles of kWideRows (at most wide_tiles a head); their tokens in `parts` parts, with
// parts > 1 in wide_bytes(tiles * heads) of workspace.
constexpr int kWideRows = 128;
int64_t wide_tiles(int64_t T, int64_t group, int64_t B);
int64_t wide_bytes(int64_t items, int parts, int64_t D);
hipError_t launch_kv_attention_wide(const AttentionArgs &args, int64_t D, int few_rows, int parts,
                                    float *work, hipStream_t stream);
hipError_t launch_kv_attention(const AttentionArgs &args, int64_t D, int64_t max_query,
                               int64_t max_seq, float *workspace, int64_t workspace_bytes,
                               hipStream_t stream);

}  // namespace rfq
