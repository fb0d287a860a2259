// The paged 8-bit key/value cache: argument checks and launches of its calls, and the kernels that build block tables and slots, quantise keys
// and values into the cache and read them back.  Attention: tsq_cache_rows.cu for few query rows, tsq_cache_tiles.cu for many.

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "tsq_cache.h"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

// ---- block tables and slots ----------------------------------------------------------------------

constexpr int kSlotThreads = 256;
constexpr int kSlotTokens = 4 * kSlotThreads;  // rows per CTA, as far as the grid goes by them

struct SlotParams {
  const int32_t *held, *added, *free_pages;
  int32_t *query_start, *lengths, *table, *slots, *taken;
  long long tokens;
  int32_t requests, n_free, table_pages, page_shift;
};

__device__ __forceinline__ long long warp_scan(long long v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long up = __shfl_up_sync(kFull, v, d);
    if (lane >= d) v += up;
  }
  return v;
}

// Exclusive sums of tokens and new pages over the requests, by every CTA for itself: the lengths are a few kilobytes that come out of L2, and nothing has to
// be waited for.  Then a thread per token: the request by bisection, the page from the table or, where the step begins it, from the free
// list.  The token at a page's first place also writes the table's entry; no entry is read that this call writes.
// Bound by latency: two dependent reads and a scan (64 requests), and by the slots written (262144 tokens 1 MB).
__global__ void __launch_bounds__(kSlotThreads) slots_kernel(const SlotParams p) {
  extern __shared__ int32_t s_requests[];  // [requests + 1] first token, [requests] rank of the first new page
  __shared__ long long s_tokens[kSlotThreads / 32], s_pages[kSlotThreads / 32];
  launch_dependents();
  wait_for_prior_grids();
  int32_t* const s_start = s_requests;
  int32_t* const s_rank = s_requests + p.requests + 1;
  const int P = 1 << p.page_shift;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int per = (p.requests + kSlotThreads - 1) / kSlotThreads;
  const int i0 = min(tid * per, p.requests), i1 = min(i0 + per, p.requests);
  long long n_tokens = 0, n_pages = 0;
  for (int i = i0; i < i1; ++i) {
    const long long held = max(p.held[i], 0), added = max(p.added[i], 0);
    n_tokens += added;
    n_pages += ((held + added + P - 1) >> p.page_shift) - ((held + P - 1) >> p.page_shift);
  }
  const long long in_tokens = warp_scan(n_tokens), in_pages = warp_scan(n_pages);
  if (lane == 31) {
    s_tokens[warp] = in_tokens;
    s_pages[warp] = in_pages;
  }
  __syncthreads();
  long long at = in_tokens - n_tokens, rank = in_pages - n_pages, all_tokens = 0, all_pages = 0;
#pragma unroll
  for (int w = 0; w < kSlotThreads / 32; ++w) {
    if (w < warp) {
      at += s_tokens[w];
      rank += s_pages[w];
    }
    all_tokens += s_tokens[w];
    all_pages += s_pages[w];
  }
  const long long most = 0x7fffffffll;
  for (int i = i0; i < i1; ++i) {
    const long long held = max(p.held[i], 0), added = max(p.added[i], 0);
    s_start[i] = static_cast<int32_t>(min(at, most));
    s_rank[i] = static_cast<int32_t>(min(rank, most));
    if (blockIdx.x == 0) {
      p.query_start[i] = static_cast<int32_t>(min(at, most));
      p.lengths[i] = static_cast<int32_t>(min(held + added, most));
    }
    at += added;
    rank += ((held + added + P - 1) >> p.page_shift) - ((held + P - 1) >> p.page_shift);
  }
  if (tid == 0) {
    s_start[p.requests] = static_cast<int32_t>(min(all_tokens, most));
    if (blockIdx.x == 0) {
      p.query_start[p.requests] = static_cast<int32_t>(min(all_tokens, most));
      *p.taken = static_cast<int32_t>(min(all_pages, most));
    }
  }
  __syncthreads();
  // every new token, with a row in slots or without one, and the rows behind the last request's: four neighbours for each thread, which mostly have
  // the request and often the page in common
  const long long total = s_start[p.requests], end = max(total, p.tokens);
  for (long long t0 = 4ll * (static_cast<long long>(blockIdx.x) * kSlotThreads + tid); t0 < end; t0 += 4ll * gridDim.x * kSlotThreads) {
    int32_t slot[4] = {-1, -1, -1, -1};
    if (t0 < total) {
      int lo = 0, hi = p.requests - 1;  // the last request that starts at or in front of t0: the one that has it
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (s_start[mid] <= t0) {
          lo = mid;
        } else {
          hi = mid - 1;
        }
      }
      long long held = max(p.held[lo], 0), known = -1;  // known: the entry that `page` is of
      int32_t page = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long t = t0 + k;
        if (t >= total) break;
        if (t >= s_start[lo + 1]) {
          do {
            ++lo;
          } while (t >= s_start[lo + 1]);  // below the total, so there is one
          held = max(p.held[lo], 0);
          known = -1;
        }
        const long long position = held + (t - s_start[lo]);
        const long long entry = position >> p.page_shift;
        const int place = static_cast<int>(position & (P - 1));
        if (entry != known) {
          const long long first = (held + P - 1) >> p.page_shift;
          known = entry;
          page = -1;
          if (entry < p.table_pages) {
            int32_t* const cell = p.table + static_cast<long long>(lo) * p.table_pages + entry;
            if (entry < first) {
              page = *cell;
            } else {
              const long long r = s_rank[lo] + (entry - first);
              page = r < p.n_free ? p.free_pages[r] : -1;
              if (place == 0) *cell = page;
            }
          }
        }
        const long long at = (static_cast<long long>(page) << p.page_shift) + place;
        if (page >= 0 && at <= most) slot[k] = static_cast<int32_t>(at);
      }
    }
    if (t0 + 4 <= p.tokens && (reinterpret_cast<uintptr_t>(p.slots) & 15u) == 0) {
      *reinterpret_cast<int4*>(p.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (t0 + k < p.tokens) p.slots[t0 + k] = slot[k];
      }
    }
  }
}

// ---- quantising into the cache -------------------------------------------------------------------

constexpr int kStoreItems = 8;            // 16-byte chunks of a thread
__host__ __device__ constexpr int store_threads(int d, int page) { return d * page / (8 * kStoreItems) > 64 ? d * page / (8 * kStoreItems) : 64; }
constexpr int kStoreBlock = 64;           // most tokens whose runs one CTA looks after
constexpr float kScaleFloor = 9.094947017729282e-13f;  // 2^-40

struct StoreParams {
  const uint16_t *k, *v;
  int8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  long long k_stride, v_stride, tokens;
  const int32_t* slots;
  int32_t heads, block;                   // tokens per CTA
  uint32_t n_slots;                       // of the cache
};

// A code from x * (1 / s), rounded to nearest even: within +-127 whatever x is, 0 for NaN (the conversion's result).
__device__ __forceinline__ uint32_t code_of(float x, float inverse) {
  return static_cast<uint32_t>(min(max(__float2int_rn(x * inverse), -127), 127)) & 0xffu;
}
__device__ __forceinline__ int signed_byte(uint32_t w, int i) { return static_cast<int>(w << (24 - 8 * i)) >> 24; }

// Four codes of one word from products in (-127.5, 127.5), each rounded by itself (mul and add on packed pairs came out as one operation): adding 1.5 * 2^23 rounds to the nearest integer (even in a tie) and leaves it in the low byte.
__device__ __forceinline__ uint32_t codes_of(uint64_t x01, uint64_t x23) {
  const uint64_t magic = pack2f(12582912.0f, 12582912.0f);
  uint32_t t0, t1, t2, t3;
  unpack2u(add2(x01, magic), t0, t1);
  unpack2u(add2(x23, magic), t2, t3);
  return __byte_perm(__byte_perm(t0, t1, 0x0040), __byte_perm(t2, t3, 0x0040), 0x5410);
}

// The larger magnitudes of two packed pairs as patterns; NaN if there is one, and with it above every number's pattern.  a holds magnitudes.
template <bool BF16>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  return Elem<BF16>::bits(__hmax2_nan(Elem<BF16>::as2(a), __habs2(Elem<BF16>::as2(b))));
}

// One CTA per head, keys or values, and block of tokens: for every run (tokens of one page) that begins in the block, the run's rows are read once into
// registers, the largest finite |x| is reduced on the 15-bit patterns, and the codes are formed from the registers.  The rows of the block are read while
// the slots are still on their way; a run that begins with the block, the usual one, then only needs the rows past it.  A page that was begun earlier has its codes
// rescaled only when the scale grows.  Block: as many tokens as leave a few CTAs per SM, a page's run at most (tsq_cache_store).
template <bool BF16, int D, int P>
__global__ void __launch_bounds__(store_threads(D, P)) store_kernel(const StoreParams p) {
  constexpr int kStoreThreads = store_threads(D, P);
  constexpr int kRowChunks = D / 8;                                    // 16-byte chunks of a row
  constexpr int kItems = (P * kRowChunks + kStoreThreads - 1) / kStoreThreads;
  __shared__ int32_t s_slot[kStoreBlock + P + 1];
  __shared__ uint32_t s_max[2][kStoreThreads / 32];
  launch_dependents();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int parts = 2 * p.heads;
  const long long t0 = static_cast<long long>(blockIdx.x / parts) * p.block;
  const int which = static_cast<int>(blockIdx.x % parts) / p.heads, head = static_cast<int>(blockIdx.x % parts) % p.heads;
  const uint16_t* const x = which ? p.v : p.k;
  const long long stride = which ? p.v_stride : p.k_stride;
  int8_t* const codes = which ? p.v_codes : p.k_codes;
  float* const scales = which ? p.v_scale : p.k_scale;
  const int early = static_cast<int>(min(static_cast<long long>(min(p.block, P)), p.tokens - t0));
  wait_for_prior_grids();
  // s_slot[1 + i] is the slot of token t0 + i, s_slot[0] that of the token in front; -1: none
  for (int i = tid; i < p.block + P + 1; i += kStoreThreads) {
    const long long t = t0 + i - 1;
    const int32_t slot = t >= 0 && t < p.tokens ? p.slots[t] : -1;
    s_slot[i] = static_cast<uint32_t>(slot) < p.n_slots ? slot : -1;
  }
  uint4 v[kItems];
  constexpr int kRowStep = kStoreThreads / kRowChunks;                 // rows from one of a thread's chunks to the next
  const int my_row = tid / kRowChunks;
  const uint16_t* const my_x = x + (t0 + my_row) * stride + head * D + tid % kRowChunks * 8;
  const auto read_rows = [&](int j, int from, int to) {  // rows from .. to of the run that begins at token j of the block
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
      const int row = my_row + it * kRowStep;
      if (row >= from && row < to) v[it] = __ldcs(reinterpret_cast<const uint4*>(my_x + (j + it * kRowStep) * stride));
    }
  };
  read_rows(0, 0, early);
  __syncthreads();
  int turn = 0;
  for (int w = 0; w < p.block; w += 32) {
    // every warp for itself, from the same slots
    const int32_t its = w + lane < p.block ? s_slot[1 + w + lane] : -1;
    const bool leads = its >= 0 && (its % P == 0 || s_slot[w + lane] != its - 1);
    for (uint32_t left = __ballot_sync(kFull, leads); left != 0; left &= left - 1) {
      const int j = w + __ffs(static_cast<int>(left)) - 1;
      const int32_t slot = s_slot[1 + j];
      const int place = slot % P;
      int n = 0;                                                       // length of the run
#pragma unroll
      for (int u = 0; u < P; u += 32) {
        const int i = u + lane;
        const uint32_t on = __ballot_sync(kFull, i < P && place + i < P && s_slot[1 + j + (i < P ? i : 0)] == slot + i);
        if (n == u) n += on == kFull ? 32 : __ffs(static_cast<int>(~on)) - 1;
      }
      const long long page_head = static_cast<long long>(slot / P) * p.heads + head;
      const float had = place > 0 ? scales[page_head] : 0.0f;
      read_rows(j, j == 0 ? early : 0, n);
      uint32_t pair = 0u;                                              // largest 15-bit patterns of the lower and the upper halves
#pragma unroll
      for (int it = 0; it < kItems; ++it) {
        if (it * kStoreThreads + tid >= n * kRowChunks) v[it] = make_uint4(0u, 0u, 0u, 0u);
        pair = larger<BF16>(larger<BF16>(larger<BF16>(larger<BF16>(pair, v[it].x), v[it].y), v[it].z), v[it].w);
      }
      uint32_t top = max(pair & 0x7fffu, (pair >> 16) & 0x7fffu);
      const bool finite = top < Elem<BF16>::kInfPattern;               // this thread's values
      if (!finite) {
        top = 0u;
#pragma unroll
        for (int it = 0; it < kItems; ++it) {
          const uint32_t words[4] = {v[it].x, v[it].y, v[it].z, v[it].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t lo = words[k] & 0x7fffu, hi = (words[k] >> 16) & 0x7fffu;
            if (lo < Elem<BF16>::kInfPattern) top = max(top, lo);
            if (hi < Elem<BF16>::kInfPattern) top = max(top, hi);
          }
        }
      }
      top = __reduce_max_sync(kFull, top);
      if (lane == 0) s_max[turn][warp] = top;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kStoreThreads / 32; ++u) top = max(top, s_max[turn][u]);
      turn ^= 1;
      const float scale = fmaxf(fmaxf(Elem<BF16>::pattern_f32(top) / 127.0f, kScaleFloor), had);
      const float inverse = 1.0f / scale;
      int8_t* const page_codes = codes + page_head * (P * D);
      // chunk it * kStoreThreads + tid of the run lies as far behind chunk tid in the page as here
      int8_t* const to = page_codes + place * D + tid * 8;
      const int chunks = n * kRowChunks;
      if (finite) {
        // |x| <= 127 s up to three roundings: the code is within +-127 without a clamp
#pragma unroll
        for (int it = 0; it < kItems; ++it) {
          if (it * kStoreThreads + tid >= chunks) continue;
          const uint32_t words[4] = {v[it].x, v[it].y, v[it].z, v[it].w};
          uint32_t out[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            out[k] = codes_of(pack2f(__fmul_rn(Elem<BF16>::lo_f32(words[2 * k]), inverse), __fmul_rn(Elem<BF16>::hi_f32(words[2 * k]), inverse)),
                              pack2f(__fmul_rn(Elem<BF16>::lo_f32(words[2 * k + 1]), inverse), __fmul_rn(Elem<BF16>::hi_f32(words[2 * k + 1]), inverse)));
          }
          *reinterpret_cast<uint2*>(to + it * (kStoreThreads * 8)) = make_uint2(out[0], out[1]);
        }
      } else {
#pragma unroll
        for (int it = 0; it < kItems; ++it) {
          if (it * kStoreThreads + tid >= chunks) continue;
          const uint32_t words[4] = {v[it].x, v[it].y, v[it].z, v[it].w};
          uint32_t out[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) out[k] = code_of(Elem<BF16>::lo_f32(words[k]), inverse) | code_of(Elem<BF16>::hi_f32(words[k]), inverse) << 8;
          *reinterpret_cast<uint2*>(to + it * (kStoreThreads * 8)) = make_uint2(out[0] | out[1] << 16, out[2] | out[3] << 16);
        }
      }
      if (place > 0 && scale != had) {
        const float ratio = had / scale;
        for (int item = tid; item < place * (D / 16); item += kStoreThreads) {
          uint4* const at = reinterpret_cast<uint4*>(page_codes) + item;
          const uint4 c = *at;
          uint32_t words[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t w4 = 0u;
#pragma unroll
            for (int b = 0; b < 4; ++b) w4 |= code_of(static_cast<float>(signed_byte(words[k], b)), ratio) << (8 * b);
            words[k] = w4;
          }
          *at = make_uint4(words[0], words[1], words[2], words[3]);
        }
      }
      if (tid == 0) scales[page_head] = scale;                         // read by every thread in front of the barrier above
    }
  }
}

// ---- reading tokens back -------------------------------------------------------------------------

constexpr int kLoadThreads = 256;
constexpr int kLoadItems = 4;             // most chunks of a thread

struct LoadParams {
  const int8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  uint16_t *k, *v;
  long long k_stride, v_stride, tokens;
  const int32_t* slots;
  int32_t heads, page_shift, block;  // tokens per CTA
  uint32_t n_slots;
};

// The four codes of a word (sign bits inverted) times a scale: 2^23 + byte less 2^23 + 128 is the code, exactly.
__device__ __forceinline__ void widen4(uint32_t u, float scale, float (&x)[4]) {
  const uint64_t less = pack2f(-8388736.0f, -8388736.0f), by = pack2f(scale, scale);
  unpack2f(mul2(add2(pack2u(__byte_perm(u, 0x4b000000u, 0x7440), __byte_perm(u, 0x4b000000u, 0x7441)), less), by), x[0], x[1]);
  unpack2f(mul2(add2(pack2u(__byte_perm(u, 0x4b000000u, 0x7442), __byte_perm(u, 0x4b000000u, 0x7443)), less), by), x[2], x[3]);
}

// A thread per 16 codes: a 16-byte load and one store of 32 bytes, a whole sector, where the rows lie on 32-byte boundaries (two stores of 16 bytes, half a sector each, otherwise; 8 codes
// and a 16-byte store per thread: 13.9 us for 8192 tokens alone, this 11.3).  A thread has a place in the token, of the keys' chunks or the values', and takes it of four
// tokens at once.  Bound by its two round trips, as much as by HBM.
template <bool BF16, int D>
__global__ void __launch_bounds__(kLoadThreads) load_kernel(const LoadParams p) {
  launch_dependents();
  const int row = p.heads * (D / 16), all = 2 * row;                       // chunks of a token's keys; of its keys and values
  const int together = max(1, kLoadThreads / all);                         // tokens that the CTA's threads have at once
  const long long t0 = static_cast<long long>(blockIdx.x) * p.block;
  const int tokens = static_cast<int>(min(static_cast<long long>(p.block), p.tokens - t0));
  const int mine = static_cast<int>(threadIdx.x) / all;                    // 0 where a token's chunks are more than the threads
  const uint32_t page_bytes = static_cast<uint32_t>(p.heads << p.page_shift) * D;  // of the keys' codes; 2^24 at most
  const int place_mask = (1 << p.page_shift) - 1;
  wait_for_prior_grids();
  if (mine >= together) return;
  for (int chunk = static_cast<int>(threadIdx.x) - mine * all; chunk < all; chunk += kLoadThreads) {
    const bool values = chunk >= row;
    const int of_row = values ? chunk - row : chunk, head = of_row / (D / 16);
    const int8_t* const codes = (values ? p.v_codes : p.k_codes) + (static_cast<long long>(head) << p.page_shift) * D + (of_row % (D / 16)) * 16;
    const float* const scales = (values ? p.v_scale : p.k_scale) + head;
    const long long stride = (values ? p.v_stride : p.k_stride) * together;  // from one of the thread's tokens to the next
    uint16_t* to = (values ? p.v : p.k) + (t0 + mine) * (values ? p.v_stride : p.k_stride) + of_row * 16;
    const bool whole = ((reinterpret_cast<uintptr_t>(to) | static_cast<uintptr_t>(2 * stride)) & 31u) == 0;  // every store of 32 bytes is aligned
    const int32_t* slots = p.slots + t0 + mine;
    for (int left = tokens - mine; left > 0; left -= kLoadItems * together) {
      uint32_t slot[kLoadItems];
      uint4 code[kLoadItems];
      float scale[kLoadItems];
#pragma unroll
      for (int n = 0; n < kLoadItems; ++n) {
        slot[n] = n * together < left ? static_cast<uint32_t>(*slots) : 0xffffffffu;
        slots += together;
      }
#pragma unroll
      for (int n = 0; n < kLoadItems; ++n) {
        code[n] = make_uint4(0u, 0u, 0u, 0u);
        scale[n] = 0.0f;
        if (slot[n] < p.n_slots) {
          const uint32_t page = slot[n] >> p.page_shift;
          code[n] = __ldcs(reinterpret_cast<const uint4*>(codes + static_cast<unsigned long long>(page) * page_bytes + (slot[n] & place_mask) * D));
          scale[n] = scales[static_cast<unsigned long long>(page) * static_cast<uint32_t>(p.heads)];
        }
      }
#pragma unroll
      for (int n = 0; n < kLoadItems; ++n) {
        if (n * together >= left) break;
        const uint32_t w[4] = {code[n].x ^ 0x80808080u, code[n].y ^ 0x80808080u, code[n].z ^ 0x80808080u, code[n].w ^ 0x80808080u};
        uint32_t out[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float x[4];
          widen4(w[k], scale[n], x);
          out[2 * k] = Elem<BF16>::pack_rn(x[0], x[1]);
          out[2 * k + 1] = Elem<BF16>::pack_rn(x[2], x[3]);
        }
        if (whole) {
          asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]), "r"(out[4]), "r"(out[5]), "r"(out[6]),
                       "r"(out[7])
                       : "memory");
        } else {
          __stcs(reinterpret_cast<uint4*>(to), make_uint4(out[0], out[1], out[2], out[3]));
          __stcs(reinterpret_cast<uint4*>(to) + 1, make_uint4(out[4], out[5], out[6], out[7]));
        }
        to += stride;
      }
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------

constexpr int kMaxSlots = 0x7fffffff;
constexpr float kMostScale = 2.0e38f;  // times log2(e) still finite

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int page_shift(int32_t page_tokens) {
  for (int s = 4; s <= 7; ++s) {
    if (page_tokens == 1 << s) return s;
  }
  return -1;
}

tsq_status_t check_cache(const tsq_cache_t* c) {
  if (!c || (c->dtype != TSQ_F16 && c->dtype != TSQ_BF16) || c->kv_heads < 1 || c->head_dim < 1 || c->page_tokens < 1 || c->pages < 1)
    return TSQ_ERR_INVALID_ARG;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return TSQ_ERR_INVALID_ARG;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return TSQ_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || page_shift(c->page_tokens) < 0) return TSQ_ERR_UNSUPPORTED;
  if (c->kv_heads > 1024) return TSQ_ERR_UNSUPPORTED;
  if (c->pages > kMaxSlots / c->page_tokens) return TSQ_ERR_INVALID_ARG;
  return TSQ_OK;
}

// Rows of `heads` heads with `stride` elements between tokens.
bool rows_fit(const void* x, long long stride, long long tokens, long long heads, int head_dim) {
  return tokens == 0 || (x && aligned(x, 16) && stride % 8 == 0 && stride >= heads * head_dim);
}

// SMs of the current device, asked for once per device.
int current_sms() {
  static std::atomic<int> known[kMaxDevices];
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= kMaxDevices) return 0;
  int n = known[device].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
    known[device].store(n, std::memory_order_relaxed);
  }
  return n;
}

// The result of a launch; a failed one leaves nothing behind for the caller's own error checks.
tsq_status_t launched(cudaError_t e) {
  if (e != cudaSuccess) {
    cudaGetLastError();
    return TSQ_ERR_CUDA;
  }
  count_launch();
  return TSQ_OK;
}

template <bool BF16, int D>
cudaError_t launch_store(const StoreParams& p, int shift, int grid, cudaStream_t stream) {
  switch (shift) {
    case 4: return launch_overlapped(store_kernel<BF16, D, 16>, grid, store_threads(D, 16), 0, stream, p);
    case 5: return launch_overlapped(store_kernel<BF16, D, 32>, grid, store_threads(D, 32), 0, stream, p);
    case 6: return launch_overlapped(store_kernel<BF16, D, 64>, grid, store_threads(D, 64), 0, stream, p);
    default: return launch_overlapped(store_kernel<BF16, D, 128>, grid, store_threads(D, 128), 0, stream, p);
  }
}

// Workspace: 16 bytes with the status, the counters of either kernel, the slots of sums.
// Which kernel: by the query rows that a key head's codes serve at most.  The row kernel reads the codes again for every 16 rows; the tile kernel takes
// 256 at once, at a step's price whether they are there or not.  us, rows / tiles (bf16, heads of 128, codes in HBM): 16 requests of 8000 keys, 8 key heads,
// 24 and 32 rows 119 / 158, 48 rows 170 / 158, 64 rows 213 / 158; 64 of 2000 keys 24 rows 123 / 176, 48 rows 176 / 178; 1 of 100000 keys 32 rows 113 / 158, 64 rows 180 / 160;
// 16 of 3000 keys, 40 key heads, 20 rows 209 / 285, 40 rows 301 / 291.
bool few_query_rows(long long max_query, int group) { return max_query * group <= kFewQueryRows; }
size_t workspace_head(int sms) { return static_cast<size_t>(align16(16ull + 4ull * sms * std::max(kRowsCtasPerSm * kRowsCounters, kTilesCounters))); }
size_t workspace_size(int sms, int head_dim, bool few) {
  const unsigned long long rows = few ? 1ull * kRowsCtasPerSm * kRowsSlots * kRowsTile : 128ull * kTilesSlots;
  return workspace_head(sms) + static_cast<size_t>(align16(4ull * rows * sms * (head_dim + 2)));
}

}  // namespace
}  // namespace tsq

using namespace tsq;

extern "C" {

tsq_status_t tsq_cache_slots(int32_t page_tokens, const int32_t* held, const int32_t* added, int32_t requests, const int32_t* free_pages, int32_t n_free,
                             int32_t* query_start, int32_t* lengths, int32_t* block_table, int32_t table_pages, int32_t* slots, int64_t tokens,
                             int32_t* taken, void* cuda_stream) {
  if (page_tokens < 1 || requests < 0 || n_free < 0 || table_pages < 0 || tokens < 0 || tokens > kMaxSlots || !query_start || !taken) return TSQ_ERR_INVALID_ARG;
  if (page_shift(page_tokens) < 0 || requests > kMaxRequests) return TSQ_ERR_UNSUPPORTED;
  if (requests > 0 && (!held || !added || !lengths || (table_pages > 0 && !block_table))) return TSQ_ERR_INVALID_ARG;
  if ((n_free > 0 && !free_pages) || (tokens > 0 && !slots)) return TSQ_ERR_INVALID_ARG;
  for (const void* a : {static_cast<const void*>(held), static_cast<const void*>(added), static_cast<const void*>(free_pages), static_cast<const void*>(query_start),
                        static_cast<const void*>(lengths), static_cast<const void*>(block_table), static_cast<const void*>(slots), static_cast<const void*>(taken)}) {
    if (!aligned(a, 4)) return TSQ_ERR_INVALID_ARG;
  }
  SlotParams p;
  std::memset(&p, 0, sizeof p);
  p.held = held;
  p.added = added;
  p.free_pages = free_pages;
  p.query_start = query_start;
  p.lengths = lengths;
  p.table = block_table;
  p.slots = slots;
  p.taken = taken;
  p.tokens = tokens;
  p.requests = requests;
  p.n_free = n_free;
  p.table_pages = table_pages;
  p.page_shift = page_shift(page_tokens);
  const size_t smem = 4ull * (2ull * static_cast<size_t>(requests) + 1ull);
  static std::atomic<unsigned long long> done{0};
  if (smem > 48 * 1024) {
    const cudaError_t e = allow_shared(slots_kernel, 4 * (2 * kMaxRequests + 1), done);
    if (e != cudaSuccess) return launched(e);
  }
  const int grid = tokens > 0 ? static_cast<int>((tokens + kSlotTokens - 1) / kSlotTokens) : 1;
  return launched(launch_overlapped(slots_kernel, grid, kSlotThreads, smem, static_cast<cudaStream_t>(cuda_stream), p));
}

tsq_status_t tsq_cache_store(const tsq_cache_t* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t tokens, const int32_t* slots,
                             void* cuda_stream) {
  const tsq_status_t fine = check_cache(cache);
  if (fine != TSQ_OK) return fine;
  if (tokens < 0 || tokens > kMaxSlots || (tokens > 0 && (!slots || !aligned(slots, 4)))) return TSQ_ERR_INVALID_ARG;
  if (!rows_fit(k, k_stride, tokens, cache->kv_heads, cache->head_dim) || !rows_fit(v, v_stride, tokens, cache->kv_heads, cache->head_dim)) return TSQ_ERR_INVALID_ARG;
  if (tokens == 0) return TSQ_OK;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  StoreParams p;
  std::memset(&p, 0, sizeof p);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.k_codes = cache->k_codes;
  p.v_codes = cache->v_codes;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.tokens = tokens;
  p.slots = slots;
  p.heads = cache->kv_heads;
  p.n_slots = static_cast<uint32_t>(cache->pages * cache->page_tokens);
  const long long parts = 2ll * cache->kv_heads;
  int block = 1;
  while (block < kStoreBlock && tokens * parts > 8ll * sms * block) block *= 2;
  p.block = block;
  const long long grid = (tokens + block - 1) / block * parts;
  if (grid > kMaxSlots) return TSQ_ERR_UNSUPPORTED;
  const int shift = page_shift(cache->page_tokens);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = cache->dtype == TSQ_BF16;
  cudaError_t e;
  if (cache->head_dim == 128) {
    e = bf16 ? launch_store<true, 128>(p, shift, static_cast<int>(grid), st) : launch_store<false, 128>(p, shift, static_cast<int>(grid), st);
  } else {
    e = bf16 ? launch_store<true, 64>(p, shift, static_cast<int>(grid), st) : launch_store<false, 64>(p, shift, static_cast<int>(grid), st);
  }
  return launched(e);
}

tsq_status_t tsq_cache_load(const tsq_cache_t* cache, const int32_t* slots, int64_t tokens, void* k, int64_t k_stride, void* v, int64_t v_stride,
                            void* cuda_stream) {
  const tsq_status_t fine = check_cache(cache);
  if (fine != TSQ_OK) return fine;
  if (tokens < 0 || tokens > kMaxSlots || (tokens > 0 && (!slots || !aligned(slots, 4)))) return TSQ_ERR_INVALID_ARG;
  if (!rows_fit(k, k_stride, tokens, cache->kv_heads, cache->head_dim) || !rows_fit(v, v_stride, tokens, cache->kv_heads, cache->head_dim)) return TSQ_ERR_INVALID_ARG;
  if (tokens == 0) return TSQ_OK;
  LoadParams p;
  std::memset(&p, 0, sizeof p);
  p.k_codes = cache->k_codes;
  p.v_codes = cache->v_codes;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.k = static_cast<uint16_t*>(k);
  p.v = static_cast<uint16_t*>(v);
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.tokens = tokens;
  p.slots = slots;
  p.heads = cache->kv_heads;
  p.page_shift = page_shift(cache->page_tokens);
  p.n_slots = static_cast<uint32_t>(cache->pages * cache->page_tokens);
  const int row = 2 * cache->kv_heads * (cache->head_dim / 16);
  // four tokens for each thread, fewer where that would leave SMs without work
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  p.block = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kLoadItems * std::max(1, kLoadThreads / row), tokens / (2 * sms))));
  const int grid = static_cast<int>((tokens + p.block - 1) / p.block);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = cache->dtype == TSQ_BF16;
  cudaError_t e;
  if (cache->head_dim == 128) {
    e = bf16 ? launch_overlapped(load_kernel<true, 128>, grid, kLoadThreads, 0, st, p) : launch_overlapped(load_kernel<false, 128>, grid, kLoadThreads, 0, st, p);
  } else {
    e = bf16 ? launch_overlapped(load_kernel<true, 64>, grid, kLoadThreads, 0, st, p) : launch_overlapped(load_kernel<false, 64>, grid, kLoadThreads, 0, st, p);
  }
  return launched(e);
}

static tsq_status_t check_attention_sizes(const tsq_cache_t* cache, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query) {
  const tsq_status_t fine = check_cache(cache);
  if (fine != TSQ_OK) return fine;
  if (tokens < 0 || tokens > kMaxSlots || requests < 0 || max_query < 1 || q_heads < 1 || q_heads % cache->kv_heads != 0) return TSQ_ERR_INVALID_ARG;
  const int group = q_heads / cache->kv_heads;
  return group > 64 || requests > kMaxRequests || tokens * group > kMaxSlots ? TSQ_ERR_UNSUPPORTED : TSQ_OK;
}

tsq_status_t tsq_cache_workspace(const tsq_cache_t* cache, int64_t tokens, int32_t q_heads, int32_t requests, int32_t max_query, size_t* workspace_bytes) {
  if (!workspace_bytes) return TSQ_ERR_INVALID_ARG;
  const tsq_status_t fine = check_attention_sizes(cache, tokens, q_heads, requests, max_query);
  if (fine != TSQ_OK) return fine;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  *workspace_bytes = workspace_size(sms, cache->head_dim, few_query_rows(max_query, q_heads / cache->kv_heads));
  return TSQ_OK;
}

tsq_status_t tsq_cache_workspace_init(void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  if (!ws_dev || !aligned(ws_dev, 16)) return TSQ_ERR_INVALID_ARG;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  if (ws_bytes < workspace_head(sms)) return TSQ_ERR_BUFFER_TOO_SMALL;
  if (cudaMemsetAsync(ws_dev, 0, workspace_head(sms), static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) {
    cudaGetLastError();
    return TSQ_ERR_CUDA;
  }
  return TSQ_OK;
}

tsq_status_t tsq_cache_attention(const tsq_cache_t* cache, const void* q, int64_t q_stride, int32_t q_heads, int64_t tokens, const int32_t* query_start,
                                 const int32_t* lengths, int32_t requests, int32_t max_query, const int32_t* block_table, int32_t table_pages, float scale,
                                 void* out, int64_t out_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  const tsq_status_t fine = check_attention_sizes(cache, tokens, q_heads, requests, max_query);
  if (fine != TSQ_OK) return fine;
  if (table_pages < 0 || !(std::fabs(scale) <= kMostScale) || !ws_dev || !aligned(ws_dev, 16)) return TSQ_ERR_INVALID_ARG;
  if (requests > 0 && (!query_start || !lengths || (table_pages > 0 && !block_table))) return TSQ_ERR_INVALID_ARG;
  if (!aligned(query_start, 4) || !aligned(lengths, 4) || !aligned(block_table, 4)) return TSQ_ERR_INVALID_ARG;
  if (!rows_fit(q, q_stride, tokens, q_heads, cache->head_dim) || !rows_fit(out, out_stride, tokens, q_heads, cache->head_dim)) return TSQ_ERR_INVALID_ARG;
  const int sms = current_sms();
  if (sms < 1) return launched(cudaErrorInvalidDevice);
  const bool few = few_query_rows(max_query, q_heads / cache->kv_heads);
  if (ws_bytes < workspace_size(sms, cache->head_dim, few)) return TSQ_ERR_BUFFER_TOO_SMALL;
  if (requests == 0 || tokens == 0) return TSQ_OK;
  AttentionParams p;
  std::memset(&p, 0, sizeof p);
  p.q = q;
  p.out = out;
  p.query_start = query_start;
  p.lengths = lengths;
  p.table = block_table;
  p.k_codes = cache->k_codes;
  p.v_codes = cache->v_codes;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.tokens = tokens;
  p.requests = requests;
  p.pages = static_cast<int32_t>(cache->pages);
  p.page_shift = page_shift(cache->page_tokens);
  p.table_pages = table_pages;
  p.kv_heads = cache->kv_heads;
  p.group = q_heads / cache->kv_heads;
  p.max_query = max_query;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = static_cast<unsigned int*>(ws_dev);
  p.counters = p.status + 4;
  p.partials = reinterpret_cast<float*>(static_cast<unsigned char*>(ws_dev) + workspace_head(sms));
  const bool bf16 = cache->dtype == TSQ_BF16;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return launched(few ? launch_attention_rows(p, bf16, cache->head_dim, sms, st) : launch_attention_tiles(p, bf16, cache->head_dim, sms, st));
}

tsq_status_t tsq_cache_workspace_status(const void* ws_dev, uint32_t* status, void* cuda_stream) {
  if (!ws_dev || !status || !aligned(ws_dev, 16)) return TSQ_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (cudaMemcpyAsync(status, ws_dev, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) {
    cudaGetLastError();
    return TSQ_ERR_CUDA;
  }
  return TSQ_OK;
}

}  // extern "C"
