// What the files of the paged 8-bit key/value cache share: kernel parameter blocks, launchers, the conversion of codes.
#ifndef TSQ_CACHE_H_
#define TSQ_CACHE_H_

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "tsq.h"

namespace tsq {

void count_launch();  // tsq_kernel_launch_count

constexpr int kMaxRequests = 8192;

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
  const int8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  long long q_stride, out_stride, tokens;  // strides in elements
  int32_t requests, table_pages, pages, kv_heads, group, max_query;
  int32_t page_shift;                      // log2 of the page's tokens
  float scale_log2;                        // scale * log2(e)
  unsigned int* status;                    // of the workspace; not TSQ_OK: a wait ran out since it was initialised, and no call uses it
  unsigned int* counters;                  // 0 between calls, as long as the status is TSQ_OK
  float* partials;                         // sums of tiles that several CTAs have a part of
};

constexpr int kFewQueryRows = 32;
// Up to so many query rows (query heads of a key head times max_query): tiles of 8 rows, four CTAs per SM, or of 16 rows, three.  A CTA has a counter for each level of
// the sums of parts and two slots of a tile's accumulators, maxima and sums in the workspace.
constexpr int kRowsCtasPerSm = 4;            // the more of the two
constexpr int kRowsTile = 16;                // likewise
constexpr int kRowsCounters = 3, kRowsSlots = 2;
// More: tiles of 256 rows, one CTA per SM, a counter for each warp of 32 rows, four slots of 128 rows.
constexpr int kTilesRows = 256;
constexpr int kTilesCounters = 8, kTilesSlots = 4;
cudaError_t launch_attention_rows(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);
cudaError_t launch_attention_tiles(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream);

}  // namespace tsq

#endif  // TSQ_CACHE_H_
