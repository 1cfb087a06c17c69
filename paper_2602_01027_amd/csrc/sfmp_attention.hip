// Attention over the 8-bit paged cache: the calls without first tokens that stay visible.
#include "sfmp_attention.h"

using namespace sfmp;

extern "C" int sfmp_kv_attention_workspace(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t q_heads,
                                           int32_t max_rows, int32_t max_tokens, int64_t* bytes) {
  if (!bytes) return SFMP_ERR_NULL;
  if (int e = check_sizes(layout, batch, rows, q_heads, max_rows, max_tokens)) return e;
  *bytes = batch && max_rows ? workspace_up_to(layout->head_dim, layout->kv_heads, q_heads / layout->kv_heads, batch, max_rows, max_tokens) : 256;
  return SFMP_OK;
}

extern "C" int sfmp_kv_attention(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev,
                                 const float* scales_dev, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                                 const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride, int32_t max_tokens,
                                 int32_t window, float scale, void* O_dev, int64_t o_stride, float* lse_dev,
                                 void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  return attend<false>(layout, layer, codes_dev, scales_dev, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, 0, scale,
                       O_dev, o_stride, lse_dev, workspace_dev, workspace_bytes, hip_stream);
}
