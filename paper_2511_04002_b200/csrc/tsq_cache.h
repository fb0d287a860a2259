// What the files of the paged 8-bit key/value cache share: kernel parameter blocks, launchers, the conversion of codes.
#ifndef TSQ_CACHE_H_
#define TSQ_CACHE_H_

#include <cuda_runtime.h>
#include <stdint.h>

#include "tsq.h"

namespace tsq {

void count_launch();  // tsq_kernel_launch_count

constexpr int kMaxRequests = 8192;

struct AttentionParams {
  const void* q;
  void* out;
  const int32_t *query_start, *lengths, *table;
  const int8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  long long q_stride, out_stride, tokens;  // strides in elements
  int32_t requests, table_pages, pages, kv_heads, group, max_query;
  int32_t page_shift;                      // log2 of the page's tokens
  float scale_log2;                        // scale * log2(e)
  unsigned int* counters;                  // one per CTA, 0 between calls
  float* partials;                         // two slots per CTA
};

// What a call of the row kernel needs of the workspace: a counter and two slots of 16 rows of accumulators, maxima and sums for every CTA.
constexpr int kRowsCtasPerSm = 3;
constexpr int kRowsTile = 16;
inline size_t rows_slot_floats(int head_dim) { return static_cast<size_t>(kRowsTile) * (head_dim + 2); }
cudaError_t launch_attention_rows(const AttentionParams& p, bool bf16, int head_dim, int ctas, cudaStream_t stream);

}  // namespace tsq

#endif  // TSQ_CACHE_H_
