/*
 * tsq — threshold splitting (TS) + token-wise adaptive bit quantisation (TAB-Q) of an LLM
 * split-point hidden state, on one NVIDIA B200 (sm_100a).
 *
 * Method: "Memory- and Latency-Constrained Inference of Large Language Models via Adaptive
 * Split Computing", Sec. II-C.  Encode = Eq. "ts" (outliers with |x| >= tau leave, undistorted,
 * as a CSR list) followed, per token row, by Algorithm 1 (TAB-Q) built on Eq. "Proposed" (AIQ):
 * a per-token min/max range over the magnitudes, a per-token bit-width chosen from a candidate
 * list by the distortion test, and the codes packed into word-aligned bit-planes.  Decode =
 * Eq. "dequnt": unpack, (code + zero-point) * scale, outliers written back.
 *
 * Conventions for every call:
 *  - plain C ABI; every pointer is marked HOST or DEVICE; the caller owns every buffer;
 *  - tsq_encode / tsq_decode only enqueue work on `cuda_stream` (a cudaStream_t passed as
 *    void*, NULL = the default stream): they never synchronise, allocate or copy to the host;
 *  - errors are return values.  Conditions that only the GPU can see (outlier capacity
 *    exceeded, malformed blob, a bounded wait that ran out) are recorded in the blob header's
 *    `status` (encode) and in the workspace (encode and decode) and are read with
 *    tsq_blob_info / tsq_workspace_status;
 *  - device tensors are contiguous row-major [tokens x hidden], 16-bit elements, base address
 *    16-byte aligned;
 *  - arithmetic is IEEE binary32, round-to-nearest-even, true division semantics, no
 *    flush-to-zero: results are bit-identical to a scalar evaluation of the paper's formulas.
 */
#ifndef TSQ_H_
#define TSQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tsq_plan tsq_plan_t; /* opaque; host-owned; immutable after creation; may be shared by threads */

typedef enum {
  TSQ_OK = 0,
  TSQ_ERR_INVALID_ARG = 1,
  TSQ_ERR_UNSUPPORTED = 2,      /* legal for the method, declined by the GPU path (e.g. hidden % 8 != 0) */
  TSQ_ERR_BUFFER_TOO_SMALL = 3,
  TSQ_ERR_CUDA = 4,             /* a CUDA runtime call failed */
  TSQ_ERR_CORRUPT_BLOB = 5,
  TSQ_ERR_OUTLIER_OVERFLOW = 6, /* more outliers than the plan's capacity; the excess was dropped */
  TSQ_ERR_TIMEOUT = 7           /* a bounded device-side wait ran out; re-initialise the workspace */
} tsq_status_t;

typedef enum { TSQ_F16 = 0, TSQ_BF16 = 1 } tsq_dtype_t;

/*
 * Which values Eq. "Proposed" quantises.
 *   TSQ_VARIANT_MAGNITUDES     Algorithm 1 as printed: sign and magnitude are separated first, a b-bit level is
 *                              one sign bit + a (b-1)-bit code of the magnitude, Q_max = 2^(b-1) - 1.
 *   TSQ_VARIANT_SIGNED_VALUES  Eq. "Proposed" applied to the signed inliers themselves (the other reading of
 *                              Sec. II-C.2, without Algorithm 1's first two steps): min and max are those of
 *                              the signed values of T_below (outlier slots count as +0), a b-bit level is a
 *                              b-bit code, Q_max = 2^b - 1, the zero-point may be negative, no sign plane.
 * A blob records its variant (header byte bits[7]) and is decoded only by a plan of the same variant.
 */
#define TSQ_VARIANT_MAGNITUDES 0
#define TSQ_VARIANT_SIGNED_VALUES 1

typedef struct {
  size_t blob_bytes;      /* bytes of the blob buffer for `tokens` rows (capacity, not payload) */
  size_t workspace_bytes; /* bytes of the workspace the plan needs (independent of `tokens`) */
} tsq_sizes_t;

typedef struct {
  uint32_t status;        /* tsq_status_t recorded by the encoder */
  uint32_t tokens, hidden, dtype;
  uint64_t total_words;   /* 32-bit words of bit-planes in use */
  uint64_t total_outliers;
  uint64_t payload_bytes; /* bytes a sender would transmit: header + per-token fields + planes + CSR */
} tsq_info_t;

/*
 * Blob format "TSQ1" (little endian; every section starts on a 16-byte boundary; capacities are
 * those of the call's `tokens` and the plan; only the first total_words / total_outliers entries
 * of the last two sections are meaningful).  WPP = ceil(hidden / 32).
 *
 *   header   64 B  u32 magic 'TSQ1' | u32 version=1 | u32 dtype | u32 hidden | u32 tokens |
 *                  u32 n_bits | u8 bits[7] | u8 variant | f32 tau | f32 delta | u64 total_words |
 *                  u64 total_outliers | u32 status | u32 outlier_capacity
 *   bits     u8  [tokens]      chosen bit-width b* (1 sign bit + (b*-1)-bit magnitude code; signed-values
 *                              variant: a b*-bit code)
 *   scale    f32 [tokens]      AIQ scale s
 *   zp       i32 [tokens]      AIQ zero-point, restore = (code + zp) * s.  The decoder accepts 0 <= zp < 2^22
 *                              (|zp| < 2^22 in the signed-values variant) and reports any other value as
 *                              TSQ_ERR_CORRUPT_BLOB: 16-bit inputs cannot produce more (the minimum over
 *                              the scale is at most 2^11 Q_max, below 2^19), and the bound keeps code + zp
 *                              exact in binary32
 *   word_off u32 [tokens+1]    exclusive prefix sum of b* x WPP
 *   out_ptr  u32 [tokens+1]    CSR row pointers (exclusive prefix sum of per-token outlier counts)
 *   words    u32 [tokens x bmax x WPP]  token t owns b* x WPP words from word_off[t], interleaved
 *                  per group of 32 elements: word g*b* + k is plane k of elements 32g .. 32g+31,
 *                  plane 0 = sign bits of the inliers, plane 1+k = bit k of the magnitude codes;
 *                  bit i of a group's word belongs to element 32g + i; pad bits are 0.  Signed-values
 *                  variant: plane k = bit k of the code, no sign plane
 *   outl     u32 [outlier_capacity]     (column << 16) | original 16-bit pattern, columns ascending
 */

/*
 * Create a plan: parameters of TS (tau, Eq. "ts") and of TAB-Q (candidate bit-widths and the
 * distortion tolerance delta of Algorithm 1; the paper's default is delta = 0.2).
 *   out          HOST   receives the plan; destroy with tsq_plan_destroy
 *   device              CUDA device ordinal the plan's kernels will run on
 *   hidden              row length H, 8 <= H <= 65536, H % 8 == 0 (else TSQ_ERR_UNSUPPORTED)
 *   max_tokens          largest `tokens` any call will pass (>= 0); tokens * H < 2^32 and
 *                       tokens * bmax * WPP < 2^32
 *   tau                 threshold; |x| >= tau, NaN and +-Inf become outliers.  +INF disables TS
 *                       for finite values, tau <= 0 makes every element an outlier.  NaN is invalid
 *   bits         HOST   n_bits strictly increasing candidates, each in [2, 8]; 1 <= n_bits <= 7
 *   delta               tolerance on the mean absolute code distortion (may be negative: no
 *                       lower candidate is ever accepted)
 *   max_outliers        CSR capacity in entries; 0 = worst case tokens * H
 * Queries device attributes; allocates no device memory.
 */
tsq_status_t tsq_plan(tsq_plan_t **out, int device, tsq_dtype_t dtype, int32_t hidden, int64_t max_tokens,
                      float tau, const int32_t *bits, int32_t n_bits, float delta, int64_t max_outliers);

/*
 * The same with the variant chosen (TSQ_VARIANT_*; tsq_plan is this call with TSQ_VARIANT_MAGNITUDES).  Any other
 * value is TSQ_ERR_INVALID_ARG.  Every other call takes plans of either variant.
 */
tsq_status_t tsq_plan_variant(tsq_plan_t **out, int device, tsq_dtype_t dtype, int32_t hidden, int64_t max_tokens,
                              float tau, const int32_t *bits, int32_t n_bits, float delta, int64_t max_outliers,
                              int32_t variant);

/* Buffer sizes for a call with `tokens` rows (0 <= tokens <= max_tokens). `out` is HOST. */
tsq_status_t tsq_plan_sizes(const tsq_plan_t *plan, int64_t tokens, tsq_sizes_t *out);

/*
 * Zero a workspace (DEVICE, workspace_bytes, 16-byte aligned) on `cuda_stream`.  Required once
 * before the buffer's first use and after any TSQ_ERR_TIMEOUT or TSQ_ERR_CUDA; encode and decode leave it ready
 * for the next call otherwise.  One workspace serves one call at a time: calls that may overlap on the GPU
 * need separate workspaces.  A workspace that plans of different max_tokens share is to be initialised
 * through the plan with the most: it is cleared as far as that plan needs it, and a call of two kernels
 * (tsq_encode) with more rows writes no row and ends with TSQ_ERR_TIMEOUT.  (Variable-length placement, the prefix sums behind word_off and
 * out_ptr, is resolved inside the encode kernels through this buffer.)
 */
tsq_status_t tsq_workspace_init(const tsq_plan_t *plan, void *ws_dev, size_t ws_bytes, void *cuda_stream);

/*
 * Set how long the encoder's device-side waits may last before they give up with TSQ_ERR_TIMEOUT.  The
 * only such wait is for placement in calls of few rows: a row's offsets are the sums over every earlier row, and a
 * row polls the workspace until those rows have published their sizes.  (Calls of more rows go through two kernels: the second
 * starts while the first still runs and polls for rows that are being sized, but no longer than the first takes, which waits for
 * nothing: no limit is needed there, and a sound call never runs out, whatever is set here.  They end with TSQ_ERR_TIMEOUT when the
 * workspace is not as a finished call leaves it, or was initialised for fewer rows.)  `polls` counts polls of one
 * row's size: one round trip apart for the first 32, then 1 us apart.  0 restores the built-in limit of 2^20 polls (about one
 * second), which is also what tsq_workspace_init sets.  With the built-in limit a wait can only run out
 * when the workspace was not initialised, is shared by calls that overlap on the GPU, or was
 * overwritten: the limit exists so that such a mistake ends in a status instead of a hang.  With a limit
 * of a few dozen polls a sound call may time out as well.  Whatever the limit, a call whose status
 * is TSQ_OK has written every row; a call of which one wait has run out may end with TSQ_ERR_TIMEOUT
 * although every row was written.  The setting is kept in the workspace (DEVICE) and is written on
 * `cuda_stream`.
 */
tsq_status_t tsq_workspace_set_wait_limit(void *ws_dev, uint32_t polls, void *cuda_stream);

/*
 * Encode x (DEVICE, [tokens x hidden]) into blob (DEVICE, >= blob_bytes from tsq_plan_sizes,
 * 16-byte aligned): TS (Eq. "ts") + TAB-Q (Algorithm 1, token-wise) + bit-plane packing, one
 * kernel launch, or two for calls of more rows than the device has SMs (signed values: more than 8).  tokens == 0 writes an empty, valid blob.  Returns argument errors before
 * anything is enqueued.
 */
tsq_status_t tsq_encode(const tsq_plan_t *plan, const void *x_dev, int64_t tokens, void *blob_dev,
                        size_t blob_bytes, void *ws_dev, size_t ws_bytes, void *cuda_stream);

/*
 * The same encode as tsq_encode, for callers that cannot give it a workspace.  (The paper has no
 * counterpart: this is a convenience of the library.)  Some hosts of this codec are not allowed to
 * allocate device memory where they call it: code running inside a region that forbids allocation
 * (a latency-critical serving loop with a frozen memory pool, a plug-in whose embedding runtime owns
 * all device memory, a thread that must never take the allocator's lock).  For them the placement
 * scratch lives in a fixed array inside the library image instead of in a caller-allocated workspace;
 * x_dev and blob_dev are still the caller's.
 *   - Limit: the plan's max_tokens must be <= 16384 (the array is 361 KB per device, held
 *     by every device that loads the library until the process exits); larger plans are refused with
 *     TSQ_ERR_UNSUPPORTED before anything is enqueued.
 *   - The call allocates and frees nothing.  The first call on a device looks up the array's device
 *     address (a one-time host-side query with that device made current for a moment); make that
 *     first call before any stream capture begins.
 *   - Each call first clears the part of the array it uses, on `cuda_stream`, then encodes.  All calls
 *     on a device share the one array: two calls whose work may overlap on the GPU (different
 *     streams, no ordering between them) race on it and corrupt each other's placement.  Order them
 *     on one stream or with events.
 *   - Asynchronous conditions are reported in the blob header only (read them with tsq_blob_info).
 * Output, arguments and errors are otherwise those of tsq_encode.
 */
tsq_status_t tsq_encode_noalloc(const tsq_plan_t *plan, const void *x_dev, int64_t tokens, void *blob_dev,
                                size_t blob_bytes, void *cuda_stream);

/*
 * Decode blob (DEVICE) into y (DEVICE, [tokens x hidden]): Eq. "dequnt".  The kernel validates the
 * header against the plan and `tokens`, and every per-token field against the blob's capacities,
 * before using it; on a mismatch it writes nothing for that blob/row and records
 * TSQ_ERR_CORRUPT_BLOB (or the encoder's own non-zero status) in the workspace.
 */
tsq_status_t tsq_decode(const tsq_plan_t *plan, const void *blob_dev, size_t blob_bytes, int64_t tokens,
                        void *y_dev, void *ws_dev, size_t ws_bytes, void *cuda_stream);

/* Copy the blob's header to the host and summarise it. Synchronises `cuda_stream`. `out` is HOST. */
tsq_status_t tsq_blob_info(const void *blob_dev, tsq_info_t *out, void *cuda_stream);

/*
 * First asynchronous error recorded in the workspace since it was initialised (TSQ_OK if none),
 * for the encoder and for the decoder.  Synchronises `cuda_stream`.  Both outputs are HOST.
 */
tsq_status_t tsq_workspace_status(const void *ws_dev, uint32_t *encode_status, uint32_t *decode_status,
                                  void *cuda_stream);

/*
 * Host-buffer convenience calls (x_host / blob_host / y_host are HOST, ideally pinned; the *_dev
 * staging buffers are DEVICE and caller-owned, sized as for tsq_encode / tsq_decode).
 * tsq_encode_host copies x to the device, encodes, and copies back the header, the per-token
 * fields and only the used part of the planes and of the CSR list; *payload_bytes (HOST) receives
 * the number of meaningful bytes.  tsq_decode_host copies a blob produced that way to the device,
 * decodes and copies y back.  Both synchronise `cuda_stream` and return the asynchronous status.
 * Calls of 8 MB of tensor and more go in parts when the plan's device is current: the copies run on two
 * streams of the library's own, ordered behind what `cuda_stream` holds and finished when the call
 * returns.  Those streams, their events and 256 bytes of pinned host memory are made by the first such
 * call on a device (calls in flight at the same time have a set each) and kept for later calls of any
 * plan: at most four sets per device, one when the device's last plan is destroyed.
 */
tsq_status_t tsq_encode_host(const tsq_plan_t *plan, const void *x_host, int64_t tokens, void *blob_host,
                             size_t blob_bytes, uint64_t *payload_bytes, void *x_dev, void *blob_dev,
                             void *ws_dev, size_t ws_bytes, void *cuda_stream);
tsq_status_t tsq_decode_host(const tsq_plan_t *plan, const void *blob_host, size_t blob_bytes, int64_t tokens,
                             void *y_host, void *blob_dev, void *y_dev, void *ws_dev, size_t ws_bytes,
                             void *cuda_stream);

/*
 * Size and latency models around the codec (host only, plain double arithmetic, no state).  They let a caller
 * take the early-exit decisions of Algorithm 2 (send the KV cache or only the hidden state, compress harder)
 * from byte counts: the model's before compression, tsq_blob_info's payload_bytes after it.  Every function
 * returns NaN for arguments outside the stated ranges.
 *
 * tsq_model_kv_bits: Eq. "bkv" (Sec. II-B), bits of KV cache held on the edge when token w (>= 1) has reached
 *   layer `layer` (1..n_layers):  2 * sum_{k<=layer} T_w Q_k + 2 * sum_{k>layer} T_{w-1} Q_k + hd * Q_layer,
 *   with T_w = w * hd and Q_k = qa_front for k < split_layer, qa_back from the split layer on (bits per element).
 * tsq_model_io_bits: Eq. "if_total", bits of the intermediate output: the whole of Eq. "bkv" when send_kv != 0,
 *   else the hidden state alone, T_w * Q_layer.
 * tsq_model_outage: P_o(R) = 1 - exp(-(2^(R/W) - 1) / gamma) (Sec. II-D.2); rate R and bandwidth W in the same
 *   unit (bits/s and Hz), gamma the received signal-to-noise ratio (linear); all three > 0.
 * tsq_model_latency: the epsilon-outage latency  bits / R * ceil(ln(epsilon) / ln(P_o(R)))  in seconds,
 *   0 < epsilon < 1 (one transmission when P_o is 0, +Inf when it is 1).
 * tsq_model_best_rate: R* = argmin over [rate_lo, rate_hi] of g(R) = ln(1 / P_o(R)) / R, by a scan of 4096
 *   cells and golden-section refinement (the paper asks for "a simple one-dimensional search").
 */
double tsq_model_kv_bits(int64_t w, int32_t layer, int32_t n_layers, int32_t split_layer, int64_t hd, double qa_front,
                         double qa_back);
double tsq_model_io_bits(int64_t w, int32_t layer, int32_t n_layers, int32_t split_layer, int64_t hd, double qa_front,
                         double qa_back, int32_t send_kv);
double tsq_model_outage(double rate, double bandwidth, double snr);
double tsq_model_latency(double bits, double rate, double bandwidth, double snr, double epsilon);
double tsq_model_best_rate(double rate_lo, double rate_hi, double bandwidth, double snr);

/*
 * The paged 8-bit key/value cache.  (The paper counts the bits of a KV cache held at Q^a bits per element, Eq. "bkv", and the machine that takes a
 * request over goes on from it; how it is held there is this library's own.)  Keys and values are whole numbers in [-127, 127] with one scale
 * for each page of tokens and head: Eq. "Proposed" on signed values with zero-point 0, the range taken over the page instead of the token.
 *
 * A cache is described by a HOST struct that the caller fills in; the library keeps nothing of it.
 *   dtype        type of the 16-bit rows that are stored, loaded and attended with
 *   kv_heads     1 .. 1024 (more are TSQ_ERR_UNSUPPORTED)
 *   head_dim     64 or 128 (else TSQ_ERR_UNSUPPORTED)
 *   page_tokens  tokens of a page: 16, 32, 64 or 128 (else TSQ_ERR_UNSUPPORTED)
 *   pages        >= 1; pages * page_tokens < 2^31
 *   k_codes, v_codes  DEVICE, [pages][kv_heads][page_tokens][head_dim], 16-byte aligned
 *   k_scale, v_scale  DEVICE, [pages][kv_heads], value = code * scale; >= 0
 * A token's slot is page * page_tokens + its place in the page.  Rows of keys, values and queries are [tokens][heads][head_dim] with the heads of a
 * token contiguous and a stride between tokens, in elements: a multiple of 8, at least heads * head_dim (so that a part of a wider
 * tensor can be passed); their base addresses are 16-byte aligned.  Every call enqueues work on `cuda_stream`, whose device has to be current,
 * and returns argument errors before anything is enqueued.  Nothing a caller leaves in the slots, tables and lengths makes a call read or write outside
 * its arrays: a slot or a page outside the cache stands for "none".
 */
typedef struct {
  tsq_dtype_t dtype;
  int32_t kv_heads, head_dim, page_tokens;
  int64_t pages;
  int8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
} tsq_cache_t;

/*
 * What a step's other calls need, from the requests' lengths, built on the GPU.  Request i has held[i] tokens in the cache and brings added[i]
 * (both int32, DEVICE, [requests]; negative counts as 0).  0 <= requests <= 8192, more are TSQ_ERR_UNSUPPORTED.
 *   query_start  out [requests + 1]   exclusive prefix sum of added (their sum has to be below 2^31)
 *   lengths      out [requests]       held + added
 *   block_table  in/out [requests][table_pages]  entry e is the page of tokens e * page_tokens ... of the request.  The entries of the pages that
 *                the step begins are written, in the order of the requests, with free_pages[0], free_pages[1], ...; -1 once the n_free are used up.
 *                Entries in front are read, those behind left as they are; pages past table_pages are not recorded
 *   slots        out [tokens]         slot of every new token, request after request; -1 where there is no page, and in the rows behind the last
 *                request's (a batch padded to a fixed size)
 *   taken        out [1]              pages that the step begins (more than n_free: the last ones got none)
 * free_pages [n_free] DEVICE.  The call is one kernel launch, with the same arguments it gives the same results again.
 */
tsq_status_t tsq_cache_slots(int32_t page_tokens, const int32_t *held, const int32_t *added, int32_t requests,
                             const int32_t *free_pages, int32_t n_free, int32_t *query_start, int32_t *lengths,
                             int32_t *block_table, int32_t table_pages, int32_t *slots, int64_t tokens, int32_t *taken,
                             void *cuda_stream);

/*
 * Quantise a step's keys and values (DEVICE, [tokens][kv_heads][head_dim], strides as above) into the cache at slots[0 .. tokens) (DEVICE; a slot
 * outside the cache: the row is skipped).  Tokens of one page have to be neighbours at successive places, as tsq_cache_slots lays them out; a page that
 * comes twice in a call is left with undefined codes and scale.  For a run at the places o, o + 1, ... of a page, for each head and for keys and
 * values apart: a = largest |x| of the run, infinities and NaN left out; scale s = max(a / 127, 2^-40), and not below the scale that the page had if
 * o > 0; codes at the places in front of o become rint(code * (s_had / s)); the run's codes are rint(x * (1 / s)), within +-127, 0 for NaN.  Places behind
 * the run keep their codes.  The arithmetic is IEEE binary32, round-to-nearest-even.  One kernel launch.
 */
tsq_status_t tsq_cache_store(const tsq_cache_t *cache, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                             int64_t tokens, const int32_t *slots, void *cuda_stream);

/*
 * Read tokens back: row t of k and v (DEVICE, strides as above) becomes code * scale of slots[t], in binary32 and rounded once to the cache's
 * dtype; 0 for a slot outside the cache.  Slots may come in any order and more than once.  (What a cache that is handed on to another machine goes through
 * tsq_encode as.)  One kernel launch.
 */
tsq_status_t tsq_cache_load(const tsq_cache_t *cache, const int32_t *slots, int64_t tokens, void *k, int64_t k_stride,
                            void *v, int64_t v_stride, void *cuda_stream);

/*
 * Attention of a step's queries over the cache.  q and out: [tokens][q_heads][head_dim] (DEVICE, strides as above), q_heads a multiple of kv_heads, at most
 * 64 times; query head h reads key head h / (q_heads / kv_heads).  Request i owns the rows query_start[i] .. query_start[i + 1) and has lengths[i]
 * tokens in the cache, its own of this step among them; its row j is the token at position lengths[i] - n_i + j and sees the positions up to its own:
 *   out = sum_p softmax_p(scale * <q, k_p>) v_p
 * A value scale below 2^-60 counts as 2^-60; the scales of the value pages that a row sees may differ by a factor of 2^80.  A scale that is NaN makes the rows NaN that see a
 * key of its page and head, and no others; negative ones are not allowed: what the rows that see them come out as is undefined.
 * Rows that see no key (n_i > lengths[i]) are written as zeros, rows behind the last request's are left as they were.  Scores, the softmax's
 * sum and the accumulators are binary32; weights are rounded to binary16, relative to the largest of their row times its page's scale.  The products of scale * log2(e) with a
 * page's key scale, with a row's largest query and with both have to stay in binary32's range, as the scores have.  bfloat16 queries are taken in binary16 relative to the
 * largest of their row and query head: exact down to 2^-31 of it, with fewer bits below, 0 under 2^-39.
 * A page outside the cache in block_table, and what lies past table_pages, is not seen.  Codes and scales behind a request's last token are not used, whatever they hold.
 *   max_query    no request has more rows than this (>= 1); rows past it are left as they were
 *   requests     0 .. 8192, more are TSQ_ERR_UNSUPPORTED; so are tokens times q_heads / kv_heads of 2^31 and more
 *   scale        within +-2e38; 1 / sqrt(head_dim) is the usual one
 *   ws           DEVICE, of tsq_cache_workspace's size or larger, 16-byte aligned, initialised once by tsq_cache_workspace_init; one workspace
 *                serves one call at a time.  Calls of a step whose sizes are not above those that the size was asked for may share it
 * Offsets into the cache are 64-bit.  One kernel launch; the same inputs give the same bits.
 */
tsq_status_t tsq_cache_workspace(const tsq_cache_t *cache, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query,
                                 size_t *workspace_bytes);
tsq_status_t tsq_cache_workspace_init(void *ws_dev, size_t ws_bytes, void *cuda_stream);
/*
 * TSQ_OK, or TSQ_ERR_TIMEOUT if a wait inside an attention call's kernel ran out since the workspace was initialised (every wait is for the call's own work: it
 * cannot in a sound call).  The output of the call that it ran out in is undefined; calls behind it leave theirs as it was, until tsq_cache_workspace_init.
 * Synchronises `cuda_stream`; `status` is HOST.
 */
tsq_status_t tsq_cache_workspace_status(const void *ws_dev, uint32_t *status, void *cuda_stream);
tsq_status_t tsq_cache_attention(const tsq_cache_t *cache, const void *q, int64_t q_stride, int32_t q_heads, int64_t tokens,
                                 const int32_t *query_start, const int32_t *lengths, int32_t requests, int32_t max_query,
                                 const int32_t *block_table, int32_t table_pages, float scale, void *out,
                                 int64_t out_stride, void *ws_dev, size_t ws_bytes, void *cuda_stream);

/*
 * The paged 4-bit key/value cache: half the bytes of the 8-bit one for each token, with a scale and a zero-point for each token and head (the range of Eq. "Proposed" on signed values at
 * 4 bits, taken over the token's row of one head).  Pages, slots, block tables (tsq_cache_slots), strides, streams, workspaces (tsq_cache_workspace_init, tsq_cache_workspace_status) and
 * errors are those of the 8-bit cache; the differences:
 *   k_codes, v_codes  DEVICE, [pages][kv_heads][page_tokens][head_dim / 2], 16-byte aligned: two codes 0 .. 15 to a byte, the even dimension's in the lower half
 *   k_grid, v_grid    DEVICE, [pages][kv_heads][page_tokens], 16-byte aligned: the scale, a bfloat16 number >= 0, in the lower half of a word, the zero-point, a signed 16-bit number within
 *                     +-1000, in the upper half.  A code stands for (code + zero-point) * scale
 */
typedef struct {
  tsq_dtype_t dtype;
  int32_t kv_heads, head_dim, page_tokens;
  int64_t pages;
  uint8_t *k_codes, *v_codes;
  uint32_t *k_grid, *v_grid;
} tsq_cache4_t;

/*
 * Quantise a step's keys and values into the cache, as tsq_cache_store.  Rows go by themselves: slots may come in any order, and nothing but a row's own codes and words is written; a slot
 * that comes twice in a call is left with codes and word of its rows in an undefined mixture.  With lo and hi the least and the largest finite number of a row, within +-2^126 (0 where none is finite):
 *   scale  s = max((hi - lo) / 15, max(|lo|, |hi|) / 128, 2^-40), in IEEE binary32 (round-to-nearest-even), then up to the next number of seven significant bits
 *   zero-point z = round(lo / s); codes max(0, min(15, round(x / s) - z)), infinities the last or the first, NaN 0; round takes halves away from zero, quotients are exact
 * One kernel launch.
 */
tsq_status_t tsq_cache4_store(const tsq_cache4_t *cache, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                              int64_t tokens, const int32_t *slots, void *cuda_stream);

/*
 * Read tokens back, as tsq_cache_load: (code + zero-point) * scale in binary32, rounded once to the cache's dtype and not beyond its largest finite number (a scale that is NaN gives NaN); 0 for a
 * slot outside the cache.  One kernel launch.
 */
tsq_status_t tsq_cache4_load(const tsq_cache4_t *cache, const int32_t *slots, int64_t tokens, void *k, int64_t k_stride,
                             void *v, int64_t v_stride, void *cuda_stream);

/*
 * Attention of a step's queries over the cache, as tsq_cache_attention, with scales and zero-points by token.
 *   causal   1: row j of request i is the token at position lengths[i] - n_i + j and sees the positions up to its own.  0: every row of request i sees all of its lengths[i] tokens, whatever
 *            n_i is (a decoder's queries over an encoder's states, which were stored once).  Anything else is TSQ_ERR_INVALID_ARG
 * A value scale below 2^-60 counts as 2^-60 in the weights' scaling and as what it is in the value; the scales of the values that a row sees may differ by a factor of 2^80.  A token whose key or
 * value scale is NaN or infinite makes the rows NaN that see it, and no others.  Codes, scales and zero-points come in as follows.
 *   up to 48 query rows (max_query times q_heads / kv_heads)  products with codes are exact, scales and zero-points come in in binary32
 *   more   keys and values are formed in binary16, each relative to its own scale or, where 16 neighbouring tokens' scales lie within a factor of 2^4, to the largest of theirs: exactly as long as
 *          the zero-point lies in -15 .. 0 and the scale has seven significant bits; otherwise zero-point times scale is rounded to binary16, and its sum with code times scale.  Weights are rounded
 *          relative to up to 2^5 times the largest of their row times its token's scale: 2^-20 of it at the small end instead of 2^-25.  A scale of 2^120 or more counts as infinite; what a value scale
 *          is below 2^-79 is lost
 * The ranges that tsq_cache_attention asks of scale, key scales and queries hold for the tokens' key scales; queries lie within +-2^120.
 * The workspace is of tsq_cache4_workspace's size or larger; one may be shared with calls over an 8-bit cache that it is large enough for.
 */
tsq_status_t tsq_cache4_workspace(const tsq_cache4_t *cache, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query,
                                  size_t *workspace_bytes);
tsq_status_t tsq_cache4_attention(const tsq_cache4_t *cache, const void *q, int64_t q_stride, int32_t q_heads, int64_t tokens,
                                  const int32_t *query_start, const int32_t *lengths, int32_t requests, int32_t max_query,
                                  const int32_t *block_table, int32_t table_pages, float scale, int32_t causal, void *out,
                                  int64_t out_stride, void *ws_dev, size_t ws_bytes, void *cuda_stream);

/* Number of kernels the library has launched in this process (all plans, all streams). */
uint64_t tsq_kernel_launch_count(void);

void tsq_plan_destroy(tsq_plan_t *plan);
const char *tsq_status_string(tsq_status_t status);

#ifdef __cplusplus
}
#endif
#endif /* TSQ_H_ */
