// Attention over a sliding window and the first tokens.
//
// The kernels are those of sfmp_attention.h, over a list of pages that holds those of the first tokens and then those of the window: what lies
// between is neither read nor counted where the work is divided.  The mask has one more comparison per score, in pages at the edge of the window or of
// the first tokens only.  8 key heads of 128 dims and groups of 4: a token behind 20000, window 1024, 11 us; 48 sequences, window 2048, 28 us for
// 124 MB, 4.4 TB/s, and 5 us to join; a chunk of 2048 rows, window 1000, 66 us, 28 of them the products of what is seen at the rate of a large one (75 us
// in the first 15 ms of a card that was idle).
#include "sfmp_attention.h"

using namespace sfmp;

extern "C" int sfmp_kv_attention_sinks(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev,
                                       const float* scales_dev, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                                       const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride, int32_t max_tokens,
                                       int32_t window, int32_t sinks, float scale, void* O_dev, int64_t o_stride, float* lse_dev,
                                       void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  // (a window that no sequence is longer than hides nothing)
  const bool all_seen = window == 0 || (tables && window > 0 && (int64_t)window >= (int64_t)tables->table_pages * kPage);
  if (sinks == 0 || (sinks > 0 && all_seen))
    return sfmp_kv_attention(layout, layer, codes_dev, scales_dev, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, scale,
                             O_dev, o_stride, lse_dev, workspace_dev, workspace_bytes, hip_stream);
  return attend<true>(layout, layer, codes_dev, scales_dev, tables, batch, Q_dev, q_heads, dtype, q_stride, max_tokens, window, sinks, scale,
                      O_dev, o_stride, lse_dev, workspace_dev, workspace_bytes, hip_stream);
}
