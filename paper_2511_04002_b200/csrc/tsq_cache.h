// What the files of the paged key/value caches share: kernel parameter blocks, launchers, host-side checks.
#ifndef TSQ_CACHE_H_
#define TSQ_CACHE_H_

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "tsq.h"

namespace tsq {

void count_launch();  // tsq_kernel_launch_count

constexpr int kMaxRequests = 8192;

// ---- host side (tsq_cache.cu) ----
constexpr int kMaxSlots = 0x7fffffff;
bool aligned(const void* p, size_t n);
int page_shift(int32_t page_tokens);         // log2; -1: not a page size
// Rows of `heads` heads with `stride` elements between tokens.
bool rows_fit(const void* x, long long stride, long long tokens, long long heads, int head_dim);
int current_sms();                           // of the current device, asked for once per device; 0: not to be had
tsq_status_t launched(cudaError_t e);        // the result of a launch; a failed one leaves nothing behind for the caller's own error checks

// Lets a kernel have so much dynamic shared memory on the current device; asked for once per kernel and device (`done`: a bit for each of the first 64).
template <typename K>
cudaError_t allow_shared(K kernel, int bytes, std::atomic<unsigned long long>& done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = device >= 0 && device < 64 ? 1ull << device : 0ull;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

struct AttentionParams {
  const void* q;
  void* out;
  const int32_t *query_start, *lengths, *table;
  const int8_t *k_codes, *v_codes;           // 8 bits each, or two of 4 bits
  const float *k_scale, *v_scale;            // of the 8-bit cache
  const uint32_t *k_grid, *v_grid;           // of the 4-bit cache
  long long q_stride, out_stride, tokens;  // strides in elements
  int32_t requests, table_pages, pages, kv_heads, group, max_query;
  int32_t page_shift;                      // log2 of the page's tokens
  int32_t causal;                          // -1: a row sees the keys up to its own position; 0: all of its request's
  float scale_log2;                        // scale * log2(e)
  unsigned int* status;                    // of the workspace; not TSQ_OK: a wait ran out since it was initialised, and no call uses it
  unsigned int* counters;                  // 0 between calls, as long as the status is TSQ_OK
  float* partials;                         // sums of tiles that several CTAs have a part of
};

constexpr int kFewQueryRows = 32;
// Up to so many query rows (query heads of a key head times max_query; the 4-bit cache has a limit of its own): tiles of 8 rows, four CTAs per SM, or of 16 rows, three.  A CTA has a counter for each level of
// the sums of parts and two slots of a tile's accumulators, maxima and sums in the workspace.
constexpr int kRowsCtasPerSm = 4;            // the more of the two
constexpr int kRowsTile = 16;                // likewise
constexpr int kRowsCounters = 3, kRowsSlots = 2;
// More: tiles of 256 rows, one CTA per SM, a counter for each warp of 32 rows, four slots of 128 rows.
constexpr int kTilesRows = 256;
constexpr int kTilesCounters = 8, kTilesSlots = 4;
cudaError_t launch_attention_rows(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);
cudaError_t launch_attention_tiles(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);
// the same over the 4-bit cache
cudaError_t launch_attention4_rows(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);
cudaError_t launch_attention4_tiles(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);
// The arguments of an attention call over either cache but the cache itself.
struct AttentionCall {
  const void* q;
  int64_t q_stride, tokens;
  int32_t q_heads;
  const int32_t *query_start, *lengths;
  int32_t requests, max_query;
  const int32_t* block_table;
  int32_t table_pages;
  float scale;
  void* out;
  int64_t out_stride;
  void* ws_dev;
  size_t ws_bytes;
};
// check_attention: of arguments whose sizes check_attention_sizes has passed; the workspace's size is left (attention_workspace_size).  fill_attention: all parameters but those of the codes.
tsq_status_t check_attention_sizes(int32_t kv_heads, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query);
tsq_status_t check_attention(const AttentionCall& a, int head_dim);
void fill_attention(const AttentionCall& a, int32_t kv_heads, int64_t pages, int page_tokens, int sms, AttentionParams& p);
size_t attention_workspace_size(int sms, int head_dim, bool few);

}  // namespace tsq

#endif  // TSQ_CACHE_H_
