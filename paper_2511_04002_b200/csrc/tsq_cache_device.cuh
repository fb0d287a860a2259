// Device-side parts that the kernels of attention over the paged 8-bit cache share.
#ifndef TSQ_CACHE_DEVICE_CUH_
#define TSQ_CACHE_DEVICE_CUH_

#include "tsq_cache.h"
#include "tsq_device.cuh"

namespace tsq {

// Weights are 2^(score + log2 s_v - m) and the softmax's sum takes them over s_v: both have to stay in binary32's range for every page that counts.  A values' scale below
// this counts as this (tsq_cache_store's are 2^-40 at least): what its codes add is under 2^-53, and a page may lie 2^80 below another of the row before its keys leave the sum.
constexpr float kLeastScale = 8.673617379884035e-19f;  // 2^-60
// Its logarithm and its inverse.  A scale that is NaN makes the weights of its keys NaN by the logarithm, and with them the rows that see one; the inverse stays a number,
// since it also multiplies the weight 0 of rows that see none.
__device__ __forceinline__ float log2_of_scale(float s) { return s != s ? s : __log2f(fmaxf(s, kLeastScale)); }
__device__ __forceinline__ float inverse_of_scale(float s) { return 1.0f / fmaxf(s, kLeastScale); }

// A request as the kernels read it: every number is brought into the range of the arrays first.
struct Request {
  long long start;   // first row
  int rows;          // rows that are written
  int keys;          // keys that can be seen: within the table
  long long before;  // position of row 0 (negative: rows that see nothing)

  __device__ __forceinline__ int tiles(int tile, const AttentionParams& p) const {
    return static_cast<int>((static_cast<long long>(rows) * p.group + tile - 1) / tile);
  }
  __device__ __forceinline__ int key_units(int unit) const { return keys > 0 ? (keys - 1) / unit + 1 : 1; }
  // a tile counts `more` units above those of its keys
  __device__ __forceinline__ unsigned long long units(int tile, int unit, int more, const AttentionParams& p) const {
    return rows == 0 ? 0ull : static_cast<unsigned long long>(tiles(tile, p)) * static_cast<unsigned>(key_units(unit) + more) * static_cast<unsigned>(p.kv_heads);
  }
  // keys that row j sees
  __device__ __forceinline__ int seen(int j) const { return static_cast<int>(max(0ll, min(static_cast<long long>(keys), before + j + 1))); }
};

__device__ __forceinline__ Request request_of(const AttentionParams& p, int i) {
  Request r;
  const long long begin = min(max(static_cast<long long>(p.query_start[i]), 0ll), p.tokens);
  const long long end = min(max(static_cast<long long>(p.query_start[i + 1]), begin), p.tokens);
  const long long length = max(p.lengths[i], 0);
  r.start = begin;
  r.rows = static_cast<int>(min(end - begin, static_cast<long long>(p.max_query)));
  r.keys = static_cast<int>(min(min(length, static_cast<long long>(p.table_pages) << p.page_shift), 0x7ffff000ll));  // a step further stays an int
  r.before = length - (end - begin);
  return r;
}

// n * total / parts; 64-bit divisions only where the numbers need them
__device__ __forceinline__ unsigned long long scaled(unsigned int n, unsigned long long total, unsigned int parts) {
  const unsigned long long v = n * total;
  return v >> 32 ? v / parts : static_cast<unsigned int>(v) / parts;
}
// The CTA whose share [c * total / ctas, (c + 1) * total / ctas) holds `unit`.
__device__ __forceinline__ int owner_of(unsigned long long unit, unsigned long long total, unsigned int ctas) {
  const unsigned long long v = (unit + 1) * ctas - 1;
  return static_cast<int>(v >> 32 || total >> 32 ? v / total : static_cast<unsigned int>(v) / static_cast<unsigned int>(total));
}
// Counts an arrival and gives what was counted before; `most` sets the counter back to 0.  What the CTA's threads wrote in front of the barrier before this is
// visible to the thread that counts last, and behind its next barrier to its CTA.
__device__ __forceinline__ unsigned int count_arrival(unsigned int* counter, unsigned int most) {
  unsigned int before;
  asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(counter), "r"(most) : "memory");
  return before;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  uint32_t u;
  memcpy(&u, &h, sizeof u);
  return u;
}

// Two codes with their sign bit inverted (code + 128) as binary16 numbers: 0x6400 + byte is 1024 + code + 128, and the difference to 1152 is exact.
__device__ __forceinline__ uint32_t less_1152(uint32_t pair) {
  const __half2 d = __hsub2(Elem<false>::as2(pair), Elem<false>::as2(0x64806480u));
  return Elem<false>::bits(d);
}
__device__ __forceinline__ uint32_t widen_lo(uint32_t u) { return less_1152(__byte_perm(u, 0x64646464u, 0x4140)); }
__device__ __forceinline__ uint32_t widen_hi(uint32_t u) { return less_1152(__byte_perm(u, 0x64646464u, 0x4342)); }

// Power of two that brings a row whose largest magnitude is `top` to just below 2^15 (2^112 at most, which brings the least bfloat16 numbers to 2^-21, a binary16 number), and the
// inverse.  Both stay in binary32's normal range; a row that is not finite is left alone.
__device__ __forceinline__ float row_power(float top, float& inverse) {
  const int e = static_cast<int>(__float_as_uint(top) >> 23);              // biased exponent; 0: below the normal range
  const int up = e < 255 ? min(14 - (e - 127), 112) : 0;
  inverse = __uint_as_float(static_cast<uint32_t>(127 - up) << 23);
  return __uint_as_float(static_cast<uint32_t>(127 + up) << 23);
}

}  // namespace tsq

#endif  // TSQ_CACHE_DEVICE_CUH_
