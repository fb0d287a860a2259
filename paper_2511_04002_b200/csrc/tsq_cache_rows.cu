// Attention over the paged 8-bit cache for few query rows per request (decode steps, drafted tokens): reads every code once.

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStepTokens = 16;              // tokens of a warp's step: within one page
constexpr int kUnitTokens = kWarps * kStepTokens;
constexpr int kFanIn = 16;                   // parts of a tile that are added up at once
constexpr int kTileUnits = 2;                // what beginning and ending a tile costs, in units

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
__device__ __forceinline__ float4 lds128f(uint32_t at) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
  return v;
}
// An 8 x 8 block of binary16 numbers, a row's two neighbours in each thread, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Over the eight threads that have the same columns.
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(kFull, v, 4));
  v = fmaxf(v, __shfl_xor_sync(kFull, v, 8));
  return fmaxf(v, __shfl_xor_sync(kFull, v, 16));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor_sync(kFull, v, 4);
  v += __shfl_xor_sync(kFull, v, 8);
  return v + __shfl_xor_sync(kFull, v, 16);
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

// The B operands of the products with the keys: thread (g, c) has of the rows row0 + 8 t + g of the tile (zeros past its `rows`) the dimensions
// c * D / 4 ... in order, four per product step.  As they lie in memory:
template <int D, int NT>
__device__ __forceinline__ void read_queries(const AttentionParams& p, const Request& r, int head, int row0, int rows, int g, int c, uint4 (&raw)[NT][D / 32]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = 8 * t + g, at = row0 + row;
    const uint16_t* const from = static_cast<const uint16_t*>(p.q) + (r.start + at / p.group) * p.q_stride +
                                 (static_cast<long long>(head) * p.group + at % p.group) * D + c * (D / 4);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) raw[t][k] = row < rows ? reinterpret_cast<const uint4*>(from)[k] : make_uint4(0u, 0u, 0u, 0u);
  }
}
// brought to binary16 by a power of two per row.  factor: the inverses for the rows 8 t + 2 c and 8 t + 2 c + 1.
template <bool BF16, int D, int NT>
__device__ __forceinline__ void scale_queries(const uint4 (&raw)[NT][D / 32], int c, uint32_t (&q)[NT][D / 16][2], float (&factor)[NT][2]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t w[D / 8];
#pragma unroll
    for (int k = 0; k < D / 32; ++k) w[4 * k] = raw[t][k].x, w[4 * k + 1] = raw[t][k].y, w[4 * k + 2] = raw[t][k].z, w[4 * k + 3] = raw[t][k].w;
    uint32_t top = 0u;
#pragma unroll
    for (int k = 0; k < D / 8; ++k) top = max(top, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    top = max(top, __shfl_xor_sync(kFull, top, 2));
    float inverse;
    const float power = row_power(Elem<BF16>::pattern_f32(top), inverse);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      q[t][k][0] = pack_half2(Elem<BF16>::lo_f32(w[2 * k]) * power, Elem<BF16>::hi_f32(w[2 * k]) * power);
      q[t][k][1] = pack_half2(Elem<BF16>::lo_f32(w[2 * k + 1]) * power, Elem<BF16>::hi_f32(w[2 * k + 1]) * power);
    }
    factor[t][0] = __shfl_sync(kFull, inverse, 8 * c);    // of the thread with g = 2 c
    factor[t][1] = __shfl_sync(kFull, inverse, 8 * c + 4);
  }
}

// Tiles of 8 query rows (NT = 1) or 16 (NT = 2).
template <int D, int NT>
struct Layout {
  static constexpr int kRows = 8 * NT;
  static constexpr int kCtasPerSm = NT == 1 ? kRowsCtasPerSm : 3;
  static constexpr int kStages = NT == 1 ? 3 : 4;        // of a warp's ring
  static constexpr int kRowChunks = D / 16;
  static constexpr int kHalf = kStepTokens * D;          // bytes of a stage's keys, and of its values
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kRing = kStages * kStage;         // of a warp
  static constexpr int kRowFloats = D + 36;              // a row of a warp's sums: four floats more behind each eighth, and four at the end
  static constexpr int kSums = kWarps * kRows * kRowFloats * 4;
  static constexpr int kMerge = kSums + kWarps * kRows * 8;
  static constexpr int kScales = kWarps * kRing > kMerge ? kWarps * kRing : kMerge;  // 64 steps' factors for each warp
  static constexpr int kBytes = kScales + kWarps * 64 * 16;
};

// Work is cut into units of 64 tokens of one (request, key head, tile of query rows), numbered in that order, and every CTA takes the same number of
// neighbouring units whatever the requests' lengths are; a tile counts kTileUnits more, for what it costs to begin and to end one.  A tile whose units lie in
// one CTA is written by it; otherwise the CTAs leave their sums in the workspace (at most two tiles of a CTA are unfinished: its first and its last) and the
// CTA that comes last adds them up in the order of the units.
//
// Within a unit each of the four warps has 16 tokens, a ring of stages of its own and its own sums; the warps meet only at a tile's end.
// Codes go from HBM to shared memory by asynchronous copies and are widened to binary16 in registers (exact).  Both products have the codes as their 16-row
// operand and the query rows as columns, eight to a product: S^T = K Q^T, O^T += V^T P^T, where P^T is S^T transposed by 8 x 8 blocks.  The order of the
// head's dimensions in the products is free: thread c of a token's four takes D / 4 neighbouring ones, so a token is read as 16-byte chunks.  Scores: q
// scaled by a power of two per row (binary16 queries exactly, bfloat16 ones down to 2^-31 of the row's largest), code products summed in binary32, times the page's
// scale.  With the values' scale s_v of the page, weights are w = 2^(score + log2 s_v - m), rounded to binary16 for the product with the values' codes, and the softmax's
// sum takes w / s_v.
// Bound by HBM where the cache is long (64 requests of 500 to 8000 tokens, 558 MB: 99 to 102 us, 5.5 TB/s), by the chain lengths -> table -> codes -> sums where it is short (one of
// 1001 tokens: 10 us).
template <bool BF16, int D, int NT>
__global__ void __launch_bounds__(kThreads, Layout<D, NT>::kCtasPerSm) attention_rows_kernel(const AttentionParams p) {
  using L = Layout<D, NT>;
  constexpr int kSteps = D / 16;                          // of the products with the keys
  constexpr int kTiles = D / 16;                          // of the sums, 16 dimensions each
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ unsigned long long s_scan[kWarps];
  __shared__ int s_found;
  __shared__ unsigned int s_status;
  __shared__ unsigned long long s_begin;
  __shared__ unsigned int s_last;
  launch_dependents();
  wait_for_prior_grids();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  const unsigned int status = *static_cast<volatile unsigned int*>(p.status);  // one thread's is used, behind a barrier: on its way with the requests

  // the CTA's share, and the request that has its first unit: every thread sums its requests' units, and the one whose sums reach past the first unit tells the others
  unsigned long long total, unit, unit_end;
  unsigned int ctas;
  {
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int i0 = min(tid * per, p.requests), i1 = min(i0 + per, p.requests);
    unsigned long long mine = 0, n = 0;
    for (int i = i0; i < i1; ++i) {
      n = request_of(p, i).units(L::kRows, kUnitTokens, kTileUnits, p);
      mine += n;
    }
    unsigned long long in = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned long long up = __shfl_up_sync(kFull, in, d);
      if (lane >= d) in += up;
    }
    if (lane == 31) s_scan[warp] = in;
    if (tid == 0) {
      s_found = 0;
      s_status = status;
      s_begin = 0;
    }
    __syncthreads();
    unsigned long long at = in - mine;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) at += s_scan[w];
      total += s_scan[w];
    }
    ctas = total < gridDim.x ? static_cast<unsigned int>(total) : gridDim.x;
    if (blockIdx.x >= ctas || s_status != TSQ_OK) return;
    unit = scaled(blockIdx.x, total, ctas);
    unit_end = scaled(blockIdx.x + 1, total, ctas);
    if (at <= unit && unit < at + mine) {
      for (int i = i0; i < i1; ++i) {
        if (per > 1) n = request_of(p, i).units(L::kRows, kUnitTokens, kTileUnits, p);
        if (unit < at + n) {
          s_found = i;
          s_begin = at;
          break;
        }
        at += n;
      }
    }
    __syncthreads();
  }
  int i = s_found;
  unsigned long long rest = unit - s_begin;               // units of request i in front of `unit`
  Request r = request_of(p, i);
  const uint32_t ring = smem_addr(smem) + warp * L::kRing, scales = smem_addr(smem) + L::kScales + warp * (64 * 16);

  while (unit < unit_end) {
    const int tiles = r.tiles(L::kRows, p), keys = r.key_units(kUnitTokens), span = keys + kTileUnits;
    const int head_tile = static_cast<int>(scaled(1, rest, span)), head = head_tile / tiles, tile = head_tile % tiles;
    const int from = static_cast<int>(rest - static_cast<unsigned long long>(head_tile) * span), upto = static_cast<int>(min(static_cast<unsigned long long>(span), from + (unit_end - unit)));
    const int k0 = max(0, from - kTileUnits), k1 = max(0, upto - kTileUnits);
    const unsigned long long tile_begin = unit - from;
    unit += upto - from;
    rest += upto - from;
    if (k1 > k0) {
      const int row0 = tile * L::kRows, rows = min(L::kRows, r.rows * p.group - row0);
      // keys that the tile's first and last rows see
      const int seen_first = r.seen(row0 / p.group), seen_last = r.seen((row0 + rows - 1) / p.group);

      // ---- the first codes on their way ----
      const int base = k0 * kUnitTokens + warp * kStepTokens;
      const int n_steps = max(0, min(k1 - k0, (seen_last - base + kUnitTokens - 1) / kUnitTokens));
      uint4 raw[NT][D / 32];
      read_queries<D, NT>(p, r, head, row0, rows, g, c, raw);
      const int32_t* const table = p.table + static_cast<long long>(i) * p.table_pages;
      // page of step 32 b + lane, -1 where there is none
      auto page_of = [&](int b) {
        const int step = 32 * b + lane;
        const int id = step < n_steps ? table[(base + step * kUnitTokens) >> p.page_shift] : -1;
        return static_cast<unsigned>(id) < static_cast<unsigned>(p.pages) ? id : -1;
      };
      // for the batch that is being worked off and the one behind it, and what is read ahead for the next
      int page_0 = page_of(0), page_1 = n_steps > 32 ? page_of(1) : -1, page_ahead = -1;
      float ks = 0.0f, vs = 1.0f;
      auto fetch_scales = [&](int page) {
        ks = page >= 0 ? p.k_scale[static_cast<long long>(page) * p.kv_heads + head] : 0.0f;
        vs = page >= 0 ? p.v_scale[static_cast<long long>(page) * p.kv_heads + head] : 1.0f;
      };
      // score factor, log2 and inverse of the values' scale of a batch's steps
      auto put_scales = [&](int b) {
        asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(scales + ((b & 1) * 32 + lane) * 16), "f"(ks * p.scale_log2), "f"(log2_of_scale(vs)), "f"(inverse_of_scale(vs)), "f"(0.0f)
                     : "memory");
      };
      auto issue = [&](int step) {
        if (step < n_steps) {
          const int id = __shfl_sync(kFull, (step >> 5) & 1 ? page_1 : page_0, step & 31);
          if (id >= 0) {
            const int token = base + step * kUnitTokens;
            const long long at = (((static_cast<long long>(id) * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1))) * D + lane * 16;
            const int8_t *const k_from = p.k_codes + at, *const v_from = p.v_codes + at;
            const uint32_t stage = ring + (step % L::kStages) * L::kStage;
#pragma unroll
            for (int n = 0; n < kStepTokens * L::kRowChunks / 32; ++n) {
              const int item = n * 32 + lane;
              const int to = placed<D>(item / L::kRowChunks, item % L::kRowChunks);
              copy16(stage + to, k_from + n * 512);
              copy16(stage + L::kHalf + to, v_from + n * 512);
            }
          }
        }
        copies_commit();
      };
      __syncthreads();                                      // the shared memory is free of the last tile's sums
#pragma unroll
      for (int s = 0; s < L::kStages - 1; ++s) issue(s);

      // ---- queries, scales ----
      fetch_scales(page_0);
      uint32_t q[NT][kSteps][2];
      float factor[NT][2];                                  // of the rows 8 t + 2 c and 8 t + 2 c + 1, whose scores this thread has
      scale_queries<BF16, D, NT>(raw, c, q, factor);
      put_scales(0);
      if (n_steps > 32) {
        fetch_scales(page_1);
        put_scales(1);
      }
      int seen[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) seen[t][h] = r.seen((row0 + min(8 * t + 2 * c + h, rows - 1)) / p.group);
      }
      __syncwarp();

      float acc[NT][kTiles][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d) acc[t][d][0] = acc[t][d][1] = acc[t][d][2] = acc[t][d][3] = 0.0f;
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.0f;
      }

      for (int step = 0; step < n_steps; ++step) {
        copies_wait<L::kStages - 2>();
        __syncwarp();
        issue(step + L::kStages - 1);
        const int id = __shfl_sync(kFull, (step >> 5) & 1 ? page_1 : page_0, step & 31);
        const float4 f = lds128f(scales + (step & 63) * 16);
        // the batch after the next takes this one's place: its pages and scales are read while this one's last steps are worked off
        if ((step & 7) == 7 && (step | 31) + 33 < n_steps) {
          if ((step & 31) == 15) page_ahead = page_of((step >> 5) + 2);
          if ((step & 31) == 23) fetch_scales(page_ahead);
        }
        if ((step & 31) == 31) {
          if (step + 33 < n_steps) {
            __syncwarp();
            put_scales(step >> 5);
          }
          if ((step >> 5) & 1) {
            page_1 = page_ahead;
          } else {
            page_0 = page_ahead;
          }
          page_ahead = -1;
        }
        if (id < 0) continue;
        const uint32_t stage = ring + (step % L::kStages) * L::kStage;
        const int token0 = base + step * kUnitTokens;

        // scores of 16 tokens and the rows
        float s[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.0f;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint4 w0 = lds128(stage + placed<D>(g, c * (D / 64) + h)), w1 = lds128(stage + placed<D>(g + 8, c * (D / 64) + h));
          const uint32_t a0[4] = {w0.x, w0.y, w0.z, w0.w}, a1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t u0 = a0[k] ^ 0x80808080u, u1 = a1[k] ^ 0x80808080u;
            const uint32_t a[4] = {widen_lo(u0), widen_lo(u1), widen_hi(u0), widen_hi(u1)};
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_16816(s[t], a, q[t][4 * h + k][0], q[t][4 * h + k][1]);
          }
        }
        bool over = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float f0 = f.x * factor[t][0], f1 = f.x * factor[t][1];
          s[t][0] = __fmaf_rn(s[t][0], f0, f.y);
          s[t][1] = __fmaf_rn(s[t][1], f1, f.y);
          s[t][2] = __fmaf_rn(s[t][2], f0, f.y);
          s[t][3] = __fmaf_rn(s[t][3], f1, f.y);
          if (token0 + kStepTokens > seen_first) {
            if (token0 + g >= seen[t][0]) s[t][0] = -INFINITY;
            if (token0 + g >= seen[t][1]) s[t][1] = -INFINITY;
            if (token0 + g + 8 >= seen[t][0]) s[t][2] = -INFINITY;
            if (token0 + g + 8 >= seen[t][1]) s[t][3] = -INFINITY;
          }
          over = over || fmaxf(s[t][0], s[t][2]) > m[t][0] + 8.0f || fmaxf(s[t][1], s[t][3]) > m[t][1] + 8.0f;
        }
        // m is a reference, not the maximum: it follows only when a score is more than 2^8 above it (a weight stays below 2^9 in binary16)
        if (__any_sync(kFull, over)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float by[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float now = fmaxf(m[t][h], column_max(fmaxf(s[t][h], s[t][2 + h])));
              by[h] = m[t][h] == -INFINITY ? 0.0f : exp2_fast(m[t][h] - now);
              m[t][h] = now;
              l[t][h] *= by[h];
            }
#pragma unroll
            for (int d = 0; d < kTiles; ++d) {
              acc[t][d][0] *= by[0];
              acc[t][d][1] *= by[1];
              acc[t][d][2] *= by[0];
              acc[t][d][3] *= by[1];
            }
          }
        }
        uint32_t w[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float ref0 = m[t][0] == -INFINITY ? 0.0f : m[t][0], ref1 = m[t][1] == -INFINITY ? 0.0f : m[t][1];
          const float x0 = exp2_fast(s[t][0] - ref0), x1 = exp2_fast(s[t][1] - ref1), x2 = exp2_fast(s[t][2] - ref0), x3 = exp2_fast(s[t][3] - ref1);
          l[t][0] = __fmaf_rn(x0 + x2, f.z, l[t][0]);
          l[t][1] = __fmaf_rn(x1 + x3, f.z, l[t][1]);
          w[t][0] = transposed(pack_half2(x0, x1));
          w[t][1] = transposed(pack_half2(x2, x3));
        }

        // values: thread (g, c) has the dimensions g * D / 8 ... of the tokens 2c, 2c + 1, 2c + 8, 2c + 9
        uint32_t v[4][D / 32];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int token = 2 * c + (t & 1) + 8 * (t >> 1);
          if constexpr (D == 128) {
            const uint4 x = lds128(stage + L::kHalf + placed<D>(token, g));
            v[t][0] = x.x, v[t][1] = x.y, v[t][2] = x.z, v[t][3] = x.w;
          } else {
            const uint2 x = lds64(stage + L::kHalf + placed<D>(token, g / 2) + 8 * (g % 2));
            v[t][0] = x.x, v[t][1] = x.y;
          }
#pragma unroll
          for (int k = 0; k < D / 32; ++k) v[t][k] ^= 0x80808080u;
        }
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          const uint32_t x0 = __byte_perm(v[0][k], v[1][k], 0x5140), x1 = __byte_perm(v[0][k], v[1][k], 0x7362);
          const uint32_t y0 = __byte_perm(v[2][k], v[3][k], 0x5140), y1 = __byte_perm(v[2][k], v[3][k], 0x7362);
          const uint32_t a0[4] = {widen_lo(x0), widen_hi(x0), widen_lo(y0), widen_hi(y0)}, a1[4] = {widen_lo(x1), widen_hi(x1), widen_lo(y1), widen_hi(y1)};
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma_16816(acc[t][2 * k], a0, w[t][0], w[t][1]);
            mma_16816(acc[t][2 * k + 1], a1, w[t][0], w[t][1]);
          }
        }
      }

      // ---- the four warps' sums ----
      copies_wait<0>();
      __syncthreads();                                      // every warp has read its stages
      float* const sums = reinterpret_cast<float*>(smem);
      float2* const stats = reinterpret_cast<float2*>(smem + L::kSums);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = warp * L::kRows + 8 * t + 2 * c + h;
          const float all = column_sum(l[t][h]);
          if (g == 0) stats[row] = make_float2(m[t][h], all);
          float* const at = sums + row * L::kRowFloats + g * (D / 8 + 4);
#pragma unroll
          for (int d = 0; d < kTiles; d += 2) *reinterpret_cast<float4*>(at + 2 * d) = make_float4(acc[t][d][h], acc[t][d][2 + h], acc[t][d + 1][h], acc[t][d + 1][2 + h]);
        }
      }
      __syncthreads();
      constexpr int kParts = kThreads / L::kRows, kDims = D / kParts;  // threads of a row, and what each has of it
      const int row = tid / kParts, d0 = tid % kParts * kDims, padded = d0 + d0 / (D / 8) * 4;
      float o[kDims], top = -INFINITY, all = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stats[w * L::kRows + row].x);
#pragma unroll
      for (int d = 0; d < kDims; ++d) o[d] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 st = stats[w * L::kRows + row];
        const float by = st.x == -INFINITY ? 0.0f : exp2_fast(st.x - top);
        all += st.y * by;
        const float* const at = sums + (w * L::kRows + row) * L::kRowFloats + padded;
#pragma unroll
        for (int d = 0; d < kDims; d += 4) {
          const float4 f4 = *reinterpret_cast<const float4*>(at + d);
          o[d] += f4.x * by;
          o[d + 1] += f4.y * by;
          o[d + 2] += f4.z * by;
          o[d + 3] += f4.w * by;
        }
      }
      bool write = true;
      if (k0 > 0 || k1 < keys) {                            // other CTAs have units of this tile
        // Parts are added up sixteen at a time by the CTA that comes last of the sixteen, their sums likewise: the order does not depend on who comes when.
        const int first = owner_of(tile_begin + kTileUnits, total, ctas), parts = owner_of(tile_begin + span - 1, total, ctas) - first + 1;
        constexpr int kSlot = L::kRows * (D + 2);
        const auto slot_of = [&](int n) { return p.partials + (2ll * (first + n) + (n == 0 ? 1 : 0)) * kSlot; };
        int part = static_cast<int>(blockIdx.x) - first;
        unsigned int* counters = p.counters;
        for (int stride = 1; stride < parts && write; stride *= kFanIn, counters += gridDim.x) {
          const int begin = part / (kFanIn * stride) * (kFanIn * stride), members = min(kFanIn, (parts - begin + stride - 1) / stride);
          if (members > 1) {
            float* const mine = slot_of(part);
            if (row < rows) {
#pragma unroll
              for (int d = 0; d < kDims; d += 4) *reinterpret_cast<float4*>(mine + row * D + d0 + d) = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
              if (d0 == 0) *reinterpret_cast<float2*>(mine + L::kRows * D + 2 * row) = make_float2(top, all);
            }
            __syncthreads();
            if (tid == 0) s_last = count_arrival(counters + first + begin, static_cast<unsigned>(members - 1)) == static_cast<unsigned>(members - 1);
            __syncthreads();
            write = s_last != 0u;
            if (write && row < rows) {
              // loads without a branch between them, so that many are on their way: past the last part its data again, with weight 0
              const auto part_at = [&](int n) { return slot_of(begin + min(n, members - 1) * stride); };
              float2 st[kFanIn];
#pragma unroll
              for (int n = 0; n < kFanIn; ++n) st[n] = __ldcg(reinterpret_cast<const float2*>(part_at(n) + L::kRows * D) + row);
              top = -INFINITY;
#pragma unroll
              for (int n = 0; n < kFanIn; ++n) {
                if (n >= members) st[n] = make_float2(-INFINITY, 0.0f);
                top = fmaxf(top, st[n].x);
              }
              all = 0.0f;
#pragma unroll
              for (int d = 0; d < kDims; ++d) o[d] = 0.0f;
              constexpr int kBatch = 64 / kDims < kFanIn ? 64 / kDims : kFanIn;
#pragma unroll
              for (int n0 = 0; n0 < kFanIn; n0 += kBatch) {
                if (n0 >= members) break;
                float4 x[kBatch][kDims / 4];
#pragma unroll
                for (int n = 0; n < kBatch; ++n) {
#pragma unroll
                  for (int d = 0; d < kDims / 4; ++d) x[n][d] = __ldcg(reinterpret_cast<const float4*>(part_at(n0 + n) + row * D + d0) + d);
                }
#pragma unroll
                for (int n = 0; n < kBatch; ++n) {
                  const float by = st[n0 + n].x == -INFINITY ? 0.0f : exp2_fast(st[n0 + n].x - top);
                  all = __fmaf_rn(st[n0 + n].y, by, all);
#pragma unroll
                  for (int d = 0; d < kDims / 4; ++d) {
                    o[4 * d] = __fmaf_rn(x[n][d].x, by, o[4 * d]);
                    o[4 * d + 1] = __fmaf_rn(x[n][d].y, by, o[4 * d + 1]);
                    o[4 * d + 2] = __fmaf_rn(x[n][d].z, by, o[4 * d + 2]);
                    o[4 * d + 3] = __fmaf_rn(x[n][d].w, by, o[4 * d + 3]);
                  }
                }
              }
            }
            __syncthreads();                                // every thread has read what the next level writes over
          }
          part = begin;
        }
      }
      write = write && row < rows;
      if (write) {
        const float by = all == 0.0f ? 0.0f : 1.0f / all;
        const int at = row0 + row;
        uint16_t* const to = static_cast<uint16_t*>(p.out) + (r.start + at / p.group) * p.out_stride + (static_cast<long long>(head) * p.group + at % p.group) * D + d0;
#pragma unroll
        for (int d = 0; d < kDims; d += 4)
          *reinterpret_cast<uint2*>(to + d) = make_uint2(Elem<BF16>::pack_rn(o[d] * by, o[d + 1] * by), Elem<BF16>::pack_rn(o[d + 2] * by, o[d + 3] * by));
      }
    }
    if (unit < unit_end && rest == r.units(L::kRows, kUnitTokens, kTileUnits, p)) {
      do {
        r = request_of(p, ++i);
      } while (r.rows == 0 && i + 1 < p.requests);
      if (r.rows == 0) break;                             // not reached while units are left
      rest = 0;
    }
  }
}

template <bool BF16, int D, int NT>
cudaError_t launch(const AttentionParams& p, int sms, cudaStream_t stream) {
  using L = Layout<D, NT>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_shared(attention_rows_kernel<BF16, D, NT>, L::kBytes, done);
  if (e != cudaSuccess) return e;
  return launch_overlapped(attention_rows_kernel<BF16, D, NT>, sms * L::kCtasPerSm, kThreads, static_cast<size_t>(L::kBytes), stream, p);
}

template <bool BF16, int D>
cudaError_t launch(const AttentionParams& p, int sms, cudaStream_t stream) {
  return static_cast<long long>(p.max_query) * p.group <= 8 ? launch<BF16, D, 1>(p, sms, stream) : launch<BF16, D, 2>(p, sms, stream);
}

}  // namespace

cudaError_t launch_attention_rows(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream) {
  if (head_dim == 128) return bf16 ? launch<true, 128>(p, sms, stream) : launch<false, 128>(p, sms, stream);
  return bf16 ? launch<true, 64>(p, sms, stream) : launch<false, 64>(p, sms, stream);
}

}  // namespace tsq
