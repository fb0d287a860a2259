// Attention over the paged 8-bit cache for few query rows per request (decode steps, drafted tokens): reads every code once.

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 4;                   // of a warp's ring
constexpr int kStepTokens = 16;              // tokens of a warp's step: within one page
constexpr int kUnitTokens = kWarps * kStepTokens;

// One m16n8k16 product, binary16 in, binary32 sums.
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ void copy16(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where the 16-byte chunk `c` of token row `t` lies in a stage: chunks change places by row, so that the four rows and two chunks that eight
// lanes read at once lie in different banks.
template <int D>
__device__ __forceinline__ int placed(int t, int c) {
  return D == 128 ? t * 128 + ((c ^ (t & 7)) << 4) : t * 64 + ((c ^ ((t >> 1) & 3)) << 4);
}

template <int D>
struct Layout {
  static constexpr int kRowChunks = D / 16;
  static constexpr int kHalf = kStepTokens * D;          // bytes of a stage's keys, and of its values
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kRing = kStages * kStage;         // of a warp
  static constexpr int kRowFloats = D + 16;              // a row of a warp's accumulators, four floats more behind each quarter
  static constexpr int kSums = kWarps * kRowsTile * kRowFloats * 4;
  static constexpr int kMerge = kSums + kWarps * kRowsTile * 8;
  static constexpr size_t kBytes = kWarps * kRing > kMerge ? kWarps * kRing : kMerge;
};

// Work is cut into units of 64 tokens of one (request, key head, tile of 16 query rows), numbered in that order, and every CTA takes the same number of
// neighbouring units whatever the requests' lengths are.  A tile whose units lie in one CTA is written by it; otherwise the CTAs leave their sums in the workspace
// (at most two tiles of a CTA are unfinished: its first and its last) and the CTA that comes last adds them up in the order of the units.
//
// Within a unit each of the four warps has 16 tokens, a ring of stages of its own and its own sums; the warps meet only at a tile's end.
// Codes go from HBM to shared memory by asynchronous copies and are widened to binary16 in registers (exact).  The order of the head's
// dimensions in the products is free: thread c of a row's four takes D / 4 neighbouring ones, so a row is read as 16-byte chunks.  Scores: q scaled by a power of two
// per row (exact), code products summed in binary32, times the page's scale.  With the values' scale s_v of the page, weights are
// w = 2^(score + log2 s_v - m), rounded to binary16 for the product with the values' codes, and the softmax's sum takes w / s_v.
template <bool BF16, int D>
__global__ void __launch_bounds__(kThreads, kRowsCtasPerSm) attention_rows_kernel(const AttentionParams p) {
  using L = Layout<D>;
  constexpr int kSteps = D / 16;                          // of the products with the keys
  constexpr int kTiles = D / 8;                           // of the accumulators, 8 dimensions each
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ unsigned long long s_scan[kWarps];
  __shared__ int s_found;
  __shared__ unsigned long long s_begin;
  __shared__ unsigned int s_last;
  launch_dependents();
  wait_for_prior_grids();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;

  // units in front of each request
  unsigned long long* const s_units = reinterpret_cast<unsigned long long*>(smem);
  unsigned long long total;
  {
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int i0 = min(tid * per, p.requests), i1 = min(i0 + per, p.requests);
    unsigned long long mine = 0;
    for (int i = i0; i < i1; ++i) mine += request_of(p, i).units(kRowsTile, kUnitTokens, p);
    unsigned long long in = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned long long up = __shfl_up_sync(kFull, in, d);
      if (lane >= d) in += up;
    }
    if (lane == 31) s_scan[warp] = in;
    __syncthreads();
    unsigned long long at = in - mine;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) at += s_scan[w];
      total += s_scan[w];
    }
    for (int i = i0; i < i1; ++i) {
      s_units[i] = at;
      at += request_of(p, i).units(kRowsTile, kUnitTokens, p);
    }
  }
  const unsigned long long ctas = total < gridDim.x ? total : gridDim.x;
  if (blockIdx.x >= ctas) return;
  unsigned long long unit = blockIdx.x * total / ctas;
  const unsigned long long unit_end = (blockIdx.x + 1) * total / ctas;
  if (tid == 0) {
    s_found = 0;
    s_begin = unit;
  }
  __syncthreads();
  for (int i = tid; i < p.requests; i += kThreads) {
    const unsigned long long begin = s_units[i], end = i + 1 < p.requests ? s_units[i + 1] : total;
    if (begin <= unit && unit < end) {
      s_found = i;
      s_begin = begin;
    }
  }
  __syncthreads();
  int i = s_found;
  unsigned long long rest = unit - s_begin;               // units of request i in front of `unit`
  Request r = request_of(p, i);
  const uint32_t ring = smem_addr(smem) + warp * L::kRing;

  while (unit < unit_end) {
    const int tiles = r.tiles(kRowsTile, p), keys = r.key_units(kUnitTokens);
    const int head_tile = static_cast<int>(rest / keys), head = head_tile / tiles, tile = head_tile % tiles;
    const int k0 = static_cast<int>(rest % keys);
    const int k1 = static_cast<int>(min(static_cast<unsigned long long>(keys), k0 + (unit_end - unit)));
    const int row0 = tile * kRowsTile, rows = min(kRowsTile, r.rows * p.group - row0);
    // keys that the tile's first and last rows, and this thread's two, see
    const int seen_first = r.seen(row0 / p.group), seen_last = r.seen((row0 + rows - 1) / p.group);
    const int seen_a = r.seen((row0 + min(g, rows - 1)) / p.group), seen_b = r.seen((row0 + min(g + 8, rows - 1)) / p.group);

    // ---- codes on their way ----
    const int base = k0 * kUnitTokens + warp * kStepTokens;
    const int n_steps = max(0, min(k1 - k0, (seen_last - base + kUnitTokens - 1) / kUnitTokens));
    const int32_t* const table = p.table + static_cast<long long>(i) * p.table_pages;
    // page, score factor, log2 and inverse of the values' scale of step 32 b + lane, for the batch b that is being worked off and the next
    int page_0 = -1, page_1 = -1;
    float fk_0 = 0.0f, fk_1 = 0.0f, lv_0 = 0.0f, lv_1 = 0.0f, iv_0 = 0.0f, iv_1 = 0.0f;
    auto fetch = [&](int b, int& page, float& fk, float& lv, float& iv) {
      const int step = 32 * b + lane, token = base + step * kUnitTokens;
      int id = -1;
      float ks = 0.0f, vs = 1.0f;
      if (step < n_steps) {
        id = table[token >> p.page_shift];
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(p.pages)) id = -1;
        if (id >= 0) {
          ks = p.k_scale[static_cast<long long>(id) * p.kv_heads + head];
          vs = fmaxf(p.v_scale[static_cast<long long>(id) * p.kv_heads + head], kLeastScale);
        }
      }
      page = id;
      fk = ks * p.scale_log2;
      lv = __log2f(vs);
      iv = 1.0f / vs;
    };
    fetch(0, page_0, fk_0, lv_0, iv_0);
    fetch(1, page_1, fk_1, lv_1, iv_1);
    auto issue = [&](int step) {
      if (step < n_steps) {
        const int id = __shfl_sync(kFull, (step >> 5) & 1 ? page_1 : page_0, step & 31);
        if (id >= 0) {
          const int token = base + step * kUnitTokens;
          const long long at = (((static_cast<long long>(id) * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1))) * D;
          const uint32_t stage = ring + (step % kStages) * L::kStage;
#pragma unroll
          for (int n = 0; n < kStepTokens * L::kRowChunks / 32; ++n) {
            const int item = n * 32 + lane;
            const int to = placed<D>(item / L::kRowChunks, item % L::kRowChunks);
            copy16(stage + to, p.k_codes + at + item * 16);
            copy16(stage + L::kHalf + to, p.v_codes + at + item * 16);
          }
        }
      }
      copies_commit();
    };
    __syncthreads();                                      // the shared memory is free of the last tile's sums, and of the unit counts
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) issue(s);

    // ---- queries ----
    uint32_t qa[kSteps][4];
    float factor_a, factor_b;
    load_queries<BF16, D>(p, r, head, row0, rows, g, c, qa, factor_a, factor_b);

    float acc[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
    float m_a = -INFINITY, m_b = -INFINITY, l_a = 0.0f, l_b = 0.0f;

    for (int step = 0; step < n_steps; ++step) {
      copies_wait<kStages - 2>();
      __syncwarp();
      issue(step + kStages - 1);
      const bool odd = ((step >> 5) & 1) != 0;
      const int id = __shfl_sync(kFull, odd ? page_1 : page_0, step & 31);
      const float f = __shfl_sync(kFull, odd ? fk_1 : fk_0, step & 31);
      const float bias = __shfl_sync(kFull, odd ? lv_1 : lv_0, step & 31);
      const float inverse = __shfl_sync(kFull, odd ? iv_1 : iv_0, step & 31);
      if ((step & 31) == 31 && step + 1 < n_steps) {      // the batch after the next takes this one's place
        if (odd) {
          fetch((step >> 5) + 2, page_1, fk_1, lv_1, iv_1);
        } else {
          fetch((step >> 5) + 2, page_0, fk_0, lv_0, iv_0);
        }
      }
      if (id < 0) continue;
      const uint32_t stage = ring + (step % kStages) * L::kStage;
      const int token0 = base + step * kUnitTokens;

      // scores of 16 rows and 16 tokens
      float s[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.0f;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint4 w = lds128(stage + placed<D>(8 * t + g, c * (D / 64) + h));
          const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t u = words[k] ^ 0x80808080u;
            mma_16816(s[t], qa[4 * h + k], widen_lo(u), widen_hi(u));
          }
        }
      }
      const float fa = f * factor_a, fb = f * factor_b;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t][0] = __fmaf_rn(s[t][0], fa, bias);
        s[t][1] = __fmaf_rn(s[t][1], fa, bias);
        s[t][2] = __fmaf_rn(s[t][2], fb, bias);
        s[t][3] = __fmaf_rn(s[t][3], fb, bias);
      }
      if (token0 + kStepTokens > seen_first) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int token = token0 + 8 * t + 2 * c;
          if (token >= seen_a) s[t][0] = -INFINITY;
          if (token + 1 >= seen_a) s[t][1] = -INFINITY;
          if (token >= seen_b) s[t][2] = -INFINITY;
          if (token + 1 >= seen_b) s[t][3] = -INFINITY;
        }
      }
      // m is a reference, not the maximum: it follows only when a score is more than 2^8 above it (a weight stays below 2^9 in binary16)
      const float top_a = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
      const float top_b = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
      if (__any_sync(kFull, top_a > m_a + 8.0f || top_b > m_b + 8.0f)) {
        const float new_a = fmaxf(m_a, quad_max(top_a)), new_b = fmaxf(m_b, quad_max(top_b));
        const float by_a = m_a == -INFINITY ? 0.0f : exp2_fast(m_a - new_a), by_b = m_b == -INFINITY ? 0.0f : exp2_fast(m_b - new_b);
        m_a = new_a;
        m_b = new_b;
        l_a *= by_a;
        l_b *= by_b;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          acc[t][0] *= by_a;
          acc[t][1] *= by_a;
          acc[t][2] *= by_b;
          acc[t][3] *= by_b;
        }
      }
      const float ref_a = m_a == -INFINITY ? 0.0f : m_a, ref_b = m_b == -INFINITY ? 0.0f : m_b;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t][0] = exp2_fast(s[t][0] - ref_a);
        s[t][1] = exp2_fast(s[t][1] - ref_a);
        s[t][2] = exp2_fast(s[t][2] - ref_b);
        s[t][3] = exp2_fast(s[t][3] - ref_b);
        l_a = __fmaf_rn(s[t][0] + s[t][1], inverse, l_a);
        l_b = __fmaf_rn(s[t][2] + s[t][3], inverse, l_b);
      }
      const uint32_t pa[4] = {pack_half2(s[0][0], s[0][1]), pack_half2(s[0][2], s[0][3]), pack_half2(s[1][0], s[1][1]), pack_half2(s[1][2], s[1][3])};

      // values: thread (g, c) has the dimensions g * D / 8 ... of the tokens 2c, 2c + 1, 2c + 8, 2c + 9
      uint32_t v[4][D / 32];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int token = 2 * c + (t & 1) + 8 * (t >> 1);
        if constexpr (D == 128) {
          const uint4 w = lds128(stage + L::kHalf + placed<D>(token, g));
          v[t][0] = w.x, v[t][1] = w.y, v[t][2] = w.z, v[t][3] = w.w;
        } else {
          const uint2 w = lds64(stage + L::kHalf + placed<D>(token, g / 2) + 8 * (g % 2));
          v[t][0] = w.x, v[t][1] = w.y;
        }
#pragma unroll
        for (int k = 0; k < D / 32; ++k) v[t][k] ^= 0x80808080u;
      }
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const uint32_t x0 = __byte_perm(v[0][k], v[1][k], 0x5140), x1 = __byte_perm(v[0][k], v[1][k], 0x7362);
        const uint32_t y0 = __byte_perm(v[2][k], v[3][k], 0x5140), y1 = __byte_perm(v[2][k], v[3][k], 0x7362);
        mma_16816(acc[4 * k], pa, widen_lo(x0), widen_lo(y0));
        mma_16816(acc[4 * k + 1], pa, widen_hi(x0), widen_hi(y0));
        mma_16816(acc[4 * k + 2], pa, widen_lo(x1), widen_lo(y1));
        mma_16816(acc[4 * k + 3], pa, widen_hi(x1), widen_hi(y1));
      }
    }
    l_a = quad_sum(l_a);
    l_b = quad_sum(l_b);

    // ---- the four warps' sums ----
    copies_wait<0>();
    __syncthreads();                                      // every warp has read its stages
    float* const sums = reinterpret_cast<float*>(smem);
    float2* const stats = reinterpret_cast<float2*>(smem + L::kSums);
    {
      float* const at = sums + (warp * kRowsTile + g) * L::kRowFloats;
#pragma unroll
      for (int col = 0; col < 2; ++col) {
        const int d0 = (2 * c + col) * (D / 8), padded = d0 + d0 / (D / 4) * 4;
#pragma unroll
        for (int t = 0; t < kTiles; t += 4) {
          *reinterpret_cast<float4*>(at + padded + t) = make_float4(acc[t][col], acc[t + 1][col], acc[t + 2][col], acc[t + 3][col]);
          *reinterpret_cast<float4*>(at + 8 * L::kRowFloats + padded + t) =
              make_float4(acc[t][2 + col], acc[t + 1][2 + col], acc[t + 2][2 + col], acc[t + 3][2 + col]);
        }
      }
      if (c == 0) {
        stats[warp * kRowsTile + g] = make_float2(m_a, l_a);
        stats[warp * kRowsTile + g + 8] = make_float2(m_b, l_b);
      }
    }
    __syncthreads();
    const int row = tid / 8, part = tid % 8, d0 = part * (D / 8), padded = d0 + d0 / (D / 4) * 4;
    float o[D / 8], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, stats[w * kRowsTile + row].x);
#pragma unroll
    for (int d = 0; d < D / 8; ++d) o[d] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 st = stats[w * kRowsTile + row];
      const float by = st.x == -INFINITY ? 0.0f : exp2_fast(st.x - m);
      l += st.y * by;
      const float* const from = sums + (w * kRowsTile + row) * L::kRowFloats + padded;
#pragma unroll
      for (int d = 0; d < D / 8; d += 4) {
        const float4 f4 = *reinterpret_cast<const float4*>(from + d);
        o[d] += f4.x * by;
        o[d + 1] += f4.y * by;
        o[d + 2] += f4.z * by;
        o[d + 3] += f4.w * by;
      }
    }
    bool write = row < rows;
    if (k0 > 0 || k1 < keys) {                            // other CTAs have units of this tile
      const unsigned long long tile_begin = unit - k0;
      const int first = static_cast<int>(((tile_begin + 1) * ctas - 1) / total), last = static_cast<int>(((tile_begin + keys) * ctas - 1) / total);
      constexpr int kSlot = kRowsTile * (D + 2);
      float* const mine = p.partials + (2ll * blockIdx.x + (k0 > 0 ? 0 : 1)) * kSlot;
      if (write) {
#pragma unroll
        for (int d = 0; d < D / 8; d += 4) *reinterpret_cast<float4*>(mine + row * D + d0 + d) = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
        if (part == 0) *reinterpret_cast<float2*>(mine + kRowsTile * D + 2 * row) = make_float2(m, l);
      }
      __threadfence();
      __syncthreads();
      if (tid == 0) s_last = atomicInc(p.counters + first, static_cast<unsigned>(last - first)) == static_cast<unsigned>(last - first);
      __syncthreads();
      write = write && s_last != 0u;
      if (write) {
        __threadfence();
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int d = 0; d < D / 8; ++d) o[d] = 0.0f;
        for (int n = first; n <= last; ++n) {
          const float* const from = p.partials + (2ll * n + (n == first ? 1 : 0)) * kSlot;
          const float2 st = __ldcg(reinterpret_cast<const float2*>(from + kRowsTile * D + 2 * row));
          const float top = fmaxf(m, st.x);
          const float by = st.x == -INFINITY ? 0.0f : exp2_fast(st.x - top), old = m == -INFINITY ? 0.0f : exp2_fast(m - top);
          m = top;
          l = l * old + st.y * by;
#pragma unroll
          for (int d = 0; d < D / 8; d += 4) {
            const float4 f4 = __ldcg(reinterpret_cast<const float4*>(from + row * D + d0 + d));
            o[d] = o[d] * old + f4.x * by;
            o[d + 1] = o[d + 1] * old + f4.y * by;
            o[d + 2] = o[d + 2] * old + f4.z * by;
            o[d + 3] = o[d + 3] * old + f4.w * by;
          }
        }
      }
    }
    if (write) {
      const float by = l == 0.0f ? 0.0f : 1.0f / l;
      const int at = row0 + row;
      uint16_t* const to = static_cast<uint16_t*>(p.out) + (r.start + at / p.group) * p.out_stride + (static_cast<long long>(head) * p.group + at % p.group) * D + d0;
      uint32_t packed[D / 16];
#pragma unroll
      for (int d = 0; d < D / 16; ++d) packed[d] = Elem<BF16>::pack_rn(o[2 * d] * by, o[2 * d + 1] * by);
#pragma unroll
      for (int d = 0; d < D / 16; d += 4) *reinterpret_cast<uint4*>(to + 2 * d) = make_uint4(packed[d], packed[d + 1], packed[d + 2], packed[d + 3]);
    }
    unit += k1 - k0;
    rest += k1 - k0;
    if (unit < unit_end && rest == r.units(kRowsTile, kUnitTokens, p)) {
      do {
        r = request_of(p, ++i);
      } while (r.rows == 0 && i + 1 < p.requests);
      if (r.rows == 0) break;                             // not reached while units are left
      rest = 0;
    }
  }
}

template <bool BF16, int D>
cudaError_t launch(const AttentionParams& p, int ctas, cudaStream_t stream) {
  static_assert(Layout<D>::kBytes >= 8 * kMaxRequests || D == 64, "unit counts fit");
  constexpr size_t smem = Layout<D>::kBytes > 8 * kMaxRequests ? Layout<D>::kBytes : 8 * kMaxRequests;
  const size_t bytes = p.requests * 8ull > Layout<D>::kBytes ? smem : Layout<D>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(attention_rows_kernel<BF16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_overlapped(attention_rows_kernel<BF16, D>, ctas, kThreads, bytes, stream, p);
}

}  // namespace

cudaError_t launch_attention_rows(const AttentionParams& p, bool bf16, int head_dim, int ctas, cudaStream_t stream) {
  if (head_dim == 128) return bf16 ? launch<true, 128>(p, ctas, stream) : launch<false, 128>(p, ctas, stream);
  return bf16 ? launch<true, 64>(p, ctas, stream) : launch<false, 64>(p, ctas, stream);
}

}  // namespace tsq
