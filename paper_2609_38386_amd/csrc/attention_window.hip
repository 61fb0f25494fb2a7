// Attention with a sliding window and sinks over bf16 pages.
#include "attention_window.h"

extern "C" int dlfp_attention_window(const dlfp_dims* dims, const dlfp_meta* meta,
                                     const int32_t* d_work, const int32_t* d_block_table,
                                     int32_t max_blocks, int32_t num_blocks, const void* q,
                                     const void* k_cache, const void* v_cache, float scale,
                                     void* out, int32_t out_dtype, void* workspace,
                                     size_t workspace_bytes, hipStream_t stream) {
  return attention_window<false>(dims, meta, d_work, d_block_table, max_blocks, num_blocks, q,
                                 k_cache, v_cache, nullptr, nullptr, scale, out, out_dtype,
                                 workspace, workspace_bytes, stream);
}
