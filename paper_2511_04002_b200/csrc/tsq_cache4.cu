// The paged 4-bit key/value cache: argument checks and launches of its calls, and the kernels that quantise keys and values into the cache and read them back.
// Attention: tsq_cache4_rows.cu for few query rows, tsq_cache_tiles.cu for many.

#include <algorithm>
#include <cstring>

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

constexpr int kMoveThreads = 128;
constexpr int kLaneNumbers = 16;          // of a row, by one thread: 32 bytes of it, 8 bytes of codes

struct Move4Params {
  uint16_t *k, *v;                        // rows: read by the store, written by the load
  uint8_t *k_codes, *v_codes;
  uint32_t *k_grid, *v_grid;
  long long k_stride, v_stride, tokens;
  const int32_t* slots;
  int32_t heads, page_shift;
  uint32_t n_slots;                       // of the cache
};

// What a thread looks after: part `part` of the row of one head, of keys or values, for the tokens first, first + step, ... of a block; neighbouring tokens are in neighbouring groups of
// threads, so that their codes and words, which lie side by side in a page, are written together.
template <int D>
struct Mine {
  static constexpr int kLanes = D / kLaneNumbers;              // threads of a row
  static constexpr int kTogether = kMoveThreads / kLanes;      // tokens at once
  int part, head;
  long long first;
  bool values;
  __device__ __forceinline__ Mine(const Move4Params& p, int items) {
    const int kinds = 2 * p.heads;
    const int kind = static_cast<int>(blockIdx.x % static_cast<unsigned>(kinds));
    values = kind >= p.heads;
    head = values ? kind - p.heads : kind;
    part = static_cast<int>(threadIdx.x) % kLanes;
    first = static_cast<long long>(blockIdx.x / static_cast<unsigned>(kinds)) * (kTogether * items) + static_cast<int>(threadIdx.x) / kLanes;
  }
};

__device__ __forceinline__ void load32(uint32_t (&w)[8], const void* at, bool whole) {
  if (whole) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(at));
  } else {
    const uint4 a = static_cast<const uint4*>(at)[0], b = static_cast<const uint4*>(at)[1];
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
}
__device__ __forceinline__ void store32(void* at, const uint32_t (&w)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
  } else {
    static_cast<uint4*>(at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    static_cast<uint4*>(at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// ---- quantising into the cache -------------------------------------------------------------------

constexpr float kMagic = 12582912.0f;     // 1.5 * 2^23: a sum with it is a whole number, which its low bits hold
constexpr int kStoreItems = 2;
template <bool BF16>
constexpr uint32_t kPlainPattern = BF16 ? 0x7e81u : 0x7c00u;  // below it: within 2^126, and finite

// Scale, zero-point and what the codes are formed with.  Halves are rounded away from zero by the product with an inverse that is 2^-20 too large, give or take the reciprocal's unit and the product's
// half one: 2^-21 to 2^-19.  x / s that is a half comes out beyond it.  Everything else stays on its side of the next half h / 2: x = X 2^a has 11 significant bits and s = S 2^b seven, so the two differ
// by 1 / (h S) of the half at least, and that is above 2^-15 as long as |x / s| <= 128 (h <= 255, S <= 127; the nearest is 127.496 beside 127.5).
struct Grid4 {
  float inverse, zero;
  uint32_t word;
  __device__ __forceinline__ Grid4(float lo, float hi) {
    lo = fmaxf(lo, -8.507059173023462e37f);                    // 2^126
    hi = fminf(hi, 8.507059173023462e37f);
    const float step = fmaxf(fmaxf(__fsub_rn(hi, lo) / 15.0f, __fmul_rn(fmaxf(fabsf(lo), fabsf(hi)), 0.0078125f)), 9.094947017729282e-13f);  // 2^-40
    const uint32_t bits = (__float_as_uint(step) + 0x1ffffu) & ~0x1ffffu;   // seven significant bits, upwards
    inverse = __fmul_rn(reciprocal(__uint_as_float(bits)), 1.00000095367431640625f);
    zero = __fsub_rn(__fmaf_rn(lo, inverse, kMagic), kMagic);
    word = bits >> 16 | static_cast<uint32_t>(static_cast<int32_t>(zero)) << 16;
  }
};

// The eight codes of four words of a row, finite numbers within its range: whole numbers 0 .. 16, the last of which counts as 15.
template <bool BF16>
__device__ __forceinline__ uint32_t nibbles_of(const uint32_t* w, uint64_t inverse, uint64_t magic) {
  uint32_t t[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack2u(fma2(pack2f(Elem<BF16>::lo_f32(w[k]), Elem<BF16>::hi_f32(w[k])), inverse, magic), t[2 * k], t[2 * k + 1]);
  uint32_t out = 0u;
#pragma unroll
  for (int k = 3; k >= 0; --k) out = mad_u32(out, 16u, __vminu2(__byte_perm(t[k], t[k + 4], 0x5410), 0x000f000fu));
  return out;
}
// The same for any number: what lies outside of the range at its ends, NaN 0.
template <bool BF16>
__device__ __forceinline__ uint32_t nibbles_of_any(const uint32_t* w, float inverse, float zero) {
  uint32_t out = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float x = k & 1 ? Elem<BF16>::hi_f32(w[k / 2]) : Elem<BF16>::lo_f32(w[k / 2]);
    const float y = fminf(fmaxf(__fmul_rn(x, inverse), -1024.0f), 1024.0f);  // NaN: -1024
    const int code = static_cast<int>(__fsub_rn(__fadd_rn(y, kMagic), kMagic) - zero);
    out |= static_cast<uint32_t>(x == x ? min(max(code, 0), 15) : 0) << (4 * k);
  }
  return out;
}

// Every row by itself, two for a thread: its numbers are read once into registers, its least and largest found on packed pairs (the largest and the negated least in one register, so that a step over the
// row's threads is one shuffle and one maximum), its codes formed by one fused operation a number.
// 8192 tokens of 8 heads of 128 (42 MB) 9.5 us, 1.5 times the copy rate's 6.5: the reads' round trip and the operations on them, of which the ALU pipe's take 4.8 us, in CTAs that follow one another.
template <bool BF16, int D>
__global__ void __launch_bounds__(kMoveThreads) store4_kernel(const Move4Params p) {
  using M = Mine<D>;
  launch_dependents();
  const M mine(p, kStoreItems);
  const uint16_t* const rows = mine.values ? p.v : p.k;
  const long long stride = mine.values ? p.v_stride : p.k_stride;
  uint8_t* const codes = mine.values ? p.v_codes : p.k_codes;
  uint32_t* const grid = mine.values ? p.v_grid : p.k_grid;
  const uint16_t* const from = rows + mine.head * D + mine.part * kLaneNumbers;
  const bool whole = ((reinterpret_cast<uintptr_t>(rows) | static_cast<uintptr_t>(2 * stride)) & 31u) == 0;
  wait_for_prior_grids();
  uint32_t x[kStoreItems][8];
  uint32_t slot[kStoreItems];
#pragma unroll
  for (int n = 0; n < kStoreItems; ++n) {
    const long long t = mine.first + n * M::kTogether;
    slot[n] = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[n][k] = 0u;
    if (t < p.tokens) {
      slot[n] = static_cast<uint32_t>(p.slots[t]);
      load32(x[n], from + t * stride, whole);
    }
  }
#pragma unroll
  for (int n = 0; n < kStoreItems; ++n) {
    uint32_t most = x[n][0], least = x[n][0];
#pragma unroll
    for (int k = 1; k < 8; ++k) {
      most = Elem<BF16>::bits(__hmax2_nan(Elem<BF16>::as2(most), Elem<BF16>::as2(x[n][k])));
      least = Elem<BF16>::bits(__hmin2_nan(Elem<BF16>::as2(least), Elem<BF16>::as2(x[n][k])));
    }
    least ^= 0x80008000u;
    uint32_t both = Elem<BF16>::bits(__hmax2_nan(Elem<BF16>::as2(__byte_perm(most, least, 0x5410)), Elem<BF16>::as2(__byte_perm(most, least, 0x7632))));
#pragma unroll
    for (int d = 1; d < M::kLanes; d *= 2) both = Elem<BF16>::bits(__hmax2_nan(Elem<BF16>::as2(both), Elem<BF16>::as2(__shfl_xor_sync(kFull, both, d))));
    const bool plain = (both & 0x7fffu) < kPlainPattern<BF16> && ((both >> 16) & 0x7fffu) < kPlainPattern<BF16>;
    float lo = -Elem<BF16>::hi_f32(both), hi = Elem<BF16>::lo_f32(both);
    const bool any = __any_sync(kFull, !plain);
    if (any) {
      lo = INFINITY;
      hi = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float a = Elem<BF16>::lo_f32(x[n][k]), b = Elem<BF16>::hi_f32(x[n][k]);
        if (fabsf(a) < INFINITY) lo = fminf(lo, a), hi = fmaxf(hi, a);
        if (fabsf(b) < INFINITY) lo = fminf(lo, b), hi = fmaxf(hi, b);
      }
#pragma unroll
      for (int d = 1; d < M::kLanes; d *= 2) {
        lo = fminf(lo, __shfl_xor_sync(kFull, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(kFull, hi, d));
      }
      if (lo > hi) lo = hi = 0.0f;
    }
    const Grid4 g(lo, hi);
    uint2 c;
    if (any) {
      c = make_uint2(nibbles_of_any<BF16>(x[n], g.inverse, g.zero), nibbles_of_any<BF16>(x[n] + 4, g.inverse, g.zero));
    } else {
      const uint64_t by = pack2f(g.inverse, g.inverse), magic = pack2f(kMagic - g.zero, kMagic - g.zero);
      c = make_uint2(nibbles_of<BF16>(x[n], by, magic), nibbles_of<BF16>(x[n] + 4, by, magic));
    }
    if (slot[n] < p.n_slots) {
      const uint32_t page = slot[n] >> p.page_shift, place = slot[n] & ((1u << p.page_shift) - 1u);
      const unsigned long long at = ((static_cast<unsigned long long>(page) * static_cast<uint32_t>(p.heads) + static_cast<uint32_t>(mine.head)) << p.page_shift) + place;
      *reinterpret_cast<uint2*>(codes + at * (D / 2) + mine.part * (kLaneNumbers / 2)) = c;
      if (mine.part == 0) grid[at] = g.word;
    }
  }
}

// ---- reading tokens back -------------------------------------------------------------------------

constexpr int kLoadItems = 2;

// (code + zero-point) * scale has 18 significant bits at most and is rounded once.  The same 8192 tokens 9.3 us: two round trips, slots and then codes, beside 34 MB of rows to write.
template <bool BF16, int D>
__global__ void __launch_bounds__(kMoveThreads) load4_kernel(const Move4Params p) {
  using M = Mine<D>;
  launch_dependents();
  const M mine(p, kLoadItems);
  uint16_t* const rows = mine.values ? p.v : p.k;
  const long long stride = mine.values ? p.v_stride : p.k_stride;
  const uint8_t* const codes = mine.values ? p.v_codes : p.k_codes;
  const uint32_t* const grid = mine.values ? p.v_grid : p.k_grid;
  uint16_t* const to = rows + mine.head * D + mine.part * kLaneNumbers;
  const bool whole = ((reinterpret_cast<uintptr_t>(rows) | static_cast<uintptr_t>(2 * stride)) & 31u) == 0;
  wait_for_prior_grids();
  uint32_t slot[kLoadItems], word[kLoadItems];
  uint2 code[kLoadItems];
#pragma unroll
  for (int n = 0; n < kLoadItems; ++n) {
    const long long t = mine.first + n * M::kTogether;
    slot[n] = t < p.tokens ? static_cast<uint32_t>(p.slots[t]) : 0xffffffffu;
  }
#pragma unroll
  for (int n = 0; n < kLoadItems; ++n) {
    word[n] = 0u;
    code[n] = make_uint2(0u, 0u);
    if (slot[n] < p.n_slots) {
      const uint32_t page = slot[n] >> p.page_shift, place = slot[n] & ((1u << p.page_shift) - 1u);
      const unsigned long long at = ((static_cast<unsigned long long>(page) * static_cast<uint32_t>(p.heads) + static_cast<uint32_t>(mine.head)) << p.page_shift) + place;
      code[n] = *reinterpret_cast<const uint2*>(codes + at * (D / 2) + mine.part * (kLaneNumbers / 2));
      word[n] = grid[at];
    }
  }
  const uint32_t largest = Elem<BF16>::kInfPattern - 1u, limit = largest | largest << 16;
#pragma unroll
  for (int n = 0; n < kLoadItems; ++n) {
    const long long t = mine.first + n * M::kTogether;
    if (t >= p.tokens) break;
    const float zero = grid_zero(word[n]), scale = grid_scale(word[n]);
    const uint64_t by = pack2f(scale, scale);
    // 0x6400 | nibble is 1024 + code, or 1024 + 16 code = 16 (64 + code) in the next four bits: the sums with the zero-point are exact in binary16
    const __half2 less_even = __float2half2_rn(zero - 1024.0f), less_odd = __float2half2_rn(zero - 64.0f), sixteenth = __float2half2_rn(0.0625f);
    uint32_t out[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t w = k ? code[n].y : code[n].x;
      float x[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {                            // the codes e and e + 4
        const uint32_t u = e < 2 ? w : w >> 8;
        const float2 c = __half22float2(e & 1 ? __hfma2(Elem<false>::as2((u & 0x00f000f0u) | 0x64006400u), sixteenth, less_odd)
                                              : __hadd2(Elem<false>::as2((u & 0x000f000fu) | 0x64006400u), less_even));
        unpack2f(mul2(pack2f(c.x, c.y), by), x[e], x[e + 4]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * k + e] = Elem<BF16>::pack_rn(x[2 * e], x[2 * e + 1]);
    }
    if (!(scale * fmaxf(fabsf(zero), fabsf(zero + 15.0f)) <= (BF16 ? 3.0e38f : 65504.0f))) {  // a code may stand for more than the type holds
#pragma unroll
      for (int k = 0; k < 8; ++k) out[k] = Elem<BF16>::bits(__hmax2_nan(__hmin2_nan(Elem<BF16>::as2(out[k]), Elem<BF16>::as2(limit)), Elem<BF16>::as2(limit | 0x80008000u)));
    }
    store32(to + t * stride, out, whole);
  }
}

// ---- host side -----------------------------------------------------------------------------------

tsq_status_t check_cache(const tsq_cache4_t* c) {
  if (!c || (c->dtype != TSQ_F16 && c->dtype != TSQ_BF16) || c->kv_heads < 1 || c->head_dim < 1 || c->page_tokens < 1 || c->pages < 1) return TSQ_ERR_INVALID_ARG;
  for (const void* a : {static_cast<const void*>(c->k_codes), static_cast<const void*>(c->v_codes), static_cast<const void*>(c->k_grid), static_cast<const void*>(c->v_grid)}) {
    if (!a || !aligned(a, 16)) return TSQ_ERR_INVALID_ARG;
  }
  if ((c->head_dim != 64 && c->head_dim != 128) || page_shift(c->page_tokens) < 0) return TSQ_ERR_UNSUPPORTED;
  if (c->kv_heads > 1024) return TSQ_ERR_UNSUPPORTED;
  if (c->pages > kMaxSlots / c->page_tokens) return TSQ_ERR_INVALID_ARG;
  return TSQ_OK;
}

tsq_status_t move_rows(const tsq_cache4_t* cache, void* k, int64_t k_stride, void* v, int64_t v_stride, int64_t tokens, const int32_t* slots, bool store, void* cuda_stream) {
  const tsq_status_t fine = check_cache(cache);
  if (fine != TSQ_OK) return fine;
  if (tokens < 0 || tokens > kMaxSlots || (tokens > 0 && (!slots || !aligned(slots, 4)))) return TSQ_ERR_INVALID_ARG;
  if (!rows_fit(k, k_stride, tokens, cache->kv_heads, cache->head_dim) || !rows_fit(v, v_stride, tokens, cache->kv_heads, cache->head_dim)) return TSQ_ERR_INVALID_ARG;
  if (tokens == 0) return TSQ_OK;
  Move4Params p;
  std::memset(&p, 0, sizeof p);
  p.k = static_cast<uint16_t*>(k);
  p.v = static_cast<uint16_t*>(v);
  p.k_codes = cache->k_codes;
  p.v_codes = cache->v_codes;
  p.k_grid = cache->k_grid;
  p.v_grid = cache->v_grid;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.tokens = tokens;
  p.slots = slots;
  p.heads = cache->kv_heads;
  p.page_shift = page_shift(cache->page_tokens);
  p.n_slots = static_cast<uint32_t>(cache->pages * cache->page_tokens);
  const int block = kMoveThreads * kLaneNumbers / cache->head_dim * (store ? kStoreItems : kLoadItems);
  const long long grid = (tokens + block - 1) / block * 2 * cache->kv_heads;
  if (grid > kMaxSlots) return TSQ_ERR_UNSUPPORTED;
  const int ctas = static_cast<int>(grid);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = cache->dtype == TSQ_BF16;
  void (*kernel)(Move4Params);
  if (cache->head_dim == 128) {
    kernel = store ? (bf16 ? store4_kernel<true, 128> : store4_kernel<false, 128>) : (bf16 ? load4_kernel<true, 128> : load4_kernel<false, 128>);
  } else {
    kernel = store ? (bf16 ? store4_kernel<true, 64> : store4_kernel<false, 64>) : (bf16 ? load4_kernel<true, 64> : load4_kernel<false, 64>);
  }
  return launched(launch_overlapped(kernel, ctas, kMoveThreads, 0, st, p));
}

// Which kernel: by the query rows that a key head's codes serve at most.  The row kernel takes the codes again for every 16 rows, the tile kernel 256 at once, at a step's price whether they
// are there or not.  us, rows / tiles, 8 key heads of 128 (of 64), bf16, fp16 within 1 %: 16 requests of 8000 keys 16 rows 51 / 144 (35 / 109), 32 rows 87 / 145 (60 / 110), 48 rows 124 / 147 (84 / 110),
// 64 rows 161 / 145 (108 / 110); 64 of 2000 keys 32 rows 96 / 150 (66 / 118), 48 rows 138 / 151 (92 / 119), 64 rows 180 / 152 (119 / 119); 1 of 100000 keys 48 rows 99 / 148 (69 / 112), 64 rows
// 125 / 149 (84 / 113), 96 rows 179 / 149 (120 / 113); 16 of 3000 keys, 40 key heads, 48 rows 240 / 254 (158 / 198), 64 rows 315 / 253 (206 / 199).
constexpr int kFewRows = 48;
bool few_query_rows(long long max_query, int group) { return max_query * group <= kFewRows; }

}  // namespace
}  // namespace tsq

using namespace tsq;

extern "C" {

tsq_status_t tsq_cache4_store(const tsq_cache4_t* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t tokens, const int32_t* slots,
                              void* cuda_stream) {
  return move_rows(cache, const_cast<void*>(k), k_stride, const_cast<void*>(v), v_stride, tokens, slots, true, cuda_stream);
}

tsq_status_t tsq_cache4_load(const tsq_cache4_t* cache, const int32_t* slots, int64_t tokens, void* k, int64_t k_stride, void* v, int64_t v_stride,
                             void* cuda_stream) {
  return move_rows(cache, k, k_stride, v, v_stride, tokens, slots, false, cuda_stream);
}

tsq_status_t tsq_cache4_workspace(const tsq_cache4_t* cache, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query, size_t* workspace_bytes) {
  if (!workspace_bytes) return TSQ_ERR_INVALID_ARG;
  tsq_status_t fine = check_cache(cache);
  if (fine == TSQ_OK) fine = check_attention_sizes(cache->kv_heads, tokens, q_heads, requests, max_query);
  if (fine != TSQ_OK) return fine;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  *workspace_bytes = attention_workspace_size(sms, cache->head_dim, few_query_rows(max_query, q_heads / cache->kv_heads));
  return TSQ_OK;
}

tsq_status_t tsq_cache4_attention(const tsq_cache4_t* cache, const void* q, int64_t q_stride, int32_t q_heads, int64_t tokens, const int32_t* query_start,
                                  const int32_t* lengths, int32_t requests, int32_t max_query, const int32_t* block_table, int32_t table_pages, float scale,
                                  int32_t causal, void* out, int64_t out_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  const AttentionCall a = {q, q_stride, tokens, q_heads, query_start, lengths, requests, max_query, block_table, table_pages, scale, out, out_stride, ws_dev, ws_bytes};
  tsq_status_t fine = check_cache(cache);
  if (fine == TSQ_OK) fine = check_attention_sizes(cache->kv_heads, tokens, q_heads, requests, max_query);
  if (fine == TSQ_OK) fine = check_attention(a, cache->head_dim);
  if (fine == TSQ_OK && causal != 0 && causal != 1) fine = TSQ_ERR_INVALID_ARG;
  if (fine != TSQ_OK) return fine;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  const bool few = few_query_rows(max_query, q_heads / cache->kv_heads);
  if (ws_bytes < attention_workspace_size(sms, cache->head_dim, few)) return TSQ_ERR_BUFFER_TOO_SMALL;
  if (requests == 0 || tokens == 0) return TSQ_OK;
  AttentionParams p;
  fill_attention(a, cache->kv_heads, cache->pages, cache->page_tokens, sms, p);
  p.causal = causal ? -1 : 0;
  p.k_codes = reinterpret_cast<const int8_t*>(cache->k_codes);
  p.v_codes = reinterpret_cast<const int8_t*>(cache->v_codes);
  p.k_grid = cache->k_grid;
  p.v_grid = cache->v_grid;
  const bool bf16 = cache->dtype == TSQ_BF16;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return launched(few ? launch_attention4_rows(p, bf16, cache->head_dim, sms, st) : launch_attention4_tiles(p, bf16, cache->head_dim, sms, st));
}

}  // extern "C"
