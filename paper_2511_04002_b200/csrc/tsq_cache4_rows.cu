// Attention over the paged 4-bit cache for few query rows per request (decode steps, drafted tokens, a decoder's step over its encoder's states): reads every code once.

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_cache_rows.cuh"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

constexpr int kWarps = kRowsWarps, kThreads = kRowsThreads;
constexpr int kStepTokens = 32;              // tokens of a warp's step, a lane each; two granules of 16, which lie in a page each
constexpr int kUnitTokens = kWarps * kStepTokens;
constexpr int kTileUnits = 1;                // what beginning and ending a tile costs, in units

__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}

// Where the 16-byte chunk `c` of token row `t` lies in a stage: chunks change places within their 128 bytes, so that the eight chunks that lanes read at once of every second
// row lie in different banks.
template <int D>
__device__ __forceinline__ int placed(int t, int c) {
  const int at = t * (D / 32) + c;
  return (at ^ (D == 128 ? ((at >> 3) & 3) << 1 : ((at >> 3) & 1) << 1)) << 4;
}

// Nibbles in bits 0 .. 3 and in bits 4 .. 7 of both halves as binary16 numbers code * 2^-20: below the normal range, but exact.  (The products take such a number at the exponent 2^-14 and cut
// what is below 2^-24 of the largest product in their sum: 2^-18 of a code here, and 2^-14 without the multiplication by 16.)
__device__ __forceinline__ uint32_t low_nibbles(uint32_t u) { return Elem<false>::bits(__hmul2(Elem<false>::as2(u & 0x000f000fu), __float2half2_rn(16.0f))); }
__device__ __forceinline__ uint32_t high_nibbles(uint32_t u) { return u & 0x00f000f0u; }

// The queries as the products with nibbles take them, brought to binary16 by a power of two per row.  Of eight dimensions the pairs (0, 4), (1, 5), (2, 6), (3, 7) go together.  factor, sum: of the rows 8 t + 2 c and 8 t + 2 c + 1, what turns sums of products into <q, code>, and the row's sum in their measure.
template <bool BF16, int D, int NT>
__device__ __forceinline__ void scale_queries(const uint4 (&raw)[NT][D / 32], int c, uint32_t (&q)[NT][D / 16][2], float (&factor)[NT][2], float (&sum)[NT][2]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t w[D / 8];
#pragma unroll
    for (int k = 0; k < D / 32; ++k) w[4 * k] = raw[t][k].x, w[4 * k + 1] = raw[t][k].y, w[4 * k + 2] = raw[t][k].z, w[4 * k + 3] = raw[t][k].w;
    uint32_t top = 0u;
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 8; ++k) top = max(top, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    top = max(top, __shfl_xor_sync(kFull, top, 2));
    float inverse;
    const float power = row_power(Elem<BF16>::pattern_f32(top), inverse);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t u = w[4 * k + h], v = w[4 * k + 2 + h];
        const float u0 = Elem<BF16>::lo_f32(u) * power, v0 = Elem<BF16>::lo_f32(v) * power, u1 = Elem<BF16>::hi_f32(u) * power, v1 = Elem<BF16>::hi_f32(v) * power;
        q[t][2 * k + h][0] = pack_half2(u0, v0);
        q[t][2 * k + h][1] = pack_half2(u1, v1);
        all += (u0 + v0) + (u1 + v1);
      }
    }
    all += __shfl_xor_sync(kFull, all, 1);
    all += __shfl_xor_sync(kFull, all, 2);
    all *= 9.5367431640625e-7f;                            // 2^-20
    inverse *= 1048576.0f;                                 // the 2^20 that a code lacks
    factor[t][0] = __shfl_sync(kFull, inverse, 8 * c);     // of the thread with g = 2 c
    factor[t][1] = __shfl_sync(kFull, inverse, 8 * c + 4);
    sum[t][0] = __shfl_sync(kFull, all, 8 * c);
    sum[t][1] = __shfl_sync(kFull, all, 8 * c + 4);
  }
}

// Tiles of 8 query rows (NT = 1) or 16 (NT = 2).
template <int D, int NT>
struct Layout {
  static constexpr int kRows = 8 * NT;
  static constexpr int kCtasPerSm = NT == 1 ? kRowsCtasPerSm : 3;
  static constexpr int kStages = NT == 1 ? 3 : 4;        // of a warp's ring
  static constexpr int kHalf = kStepTokens * D / 2;      // bytes of a stage's keys, and of its values
  static constexpr int kWords = 2 * kHalf;               // behind them: the keys' words, the values'
  static constexpr int kStage = kWords + 2 * kStepTokens * 4;
  static constexpr int kRing = kStages * kStage;         // of a warp
  static constexpr int kMerge = RowsSums<D, NT>::kBytes;
  static constexpr int kTokens = kWarps * kRing > kMerge ? kWarps * kRing : kMerge;  // a step's factors for each warp: four numbers a token, then the values' zero-points in binary16
  static constexpr int kTokenBytes = kStepTokens * 18;
  static constexpr int kBytes = kTokens + kWarps * kTokenBytes;
};

// As over the 8-bit cache (tsq_cache_rows.cu): units of neighbouring tokens of one (request, key head, tile of query rows), the same number for every CTA; the four warps have 32
// tokens of a unit each, a ring of stages and sums of their own; codes are the 16-row operand of both products.  What 4 bits change:
//
// A nibble alone in bits 4 .. 7 of a 16-bit field is the binary16 number code * 2^-20, and one in bits 0 .. 3 that by a multiplication by 16.  So a word becomes four operand registers by four
// masks, a shift and two packed products: (0, 4) and (1, 5) of its eight codes, then (2, 6) and (3, 7).  What that leaves is put right outside of the products:
//   score  = s_k (sum q c + z_k sum q)          by two operations per score, the keys' scale and zero-point by token
//   out    = (sum w c + sum w z_v) / sum p      w = p s_v rounded to binary16, as over the 8-bit cache: 2^(score + log2 s_v - m), relative to the row's largest;
//                                               the second sum is one more product, whose operand is the zero-points, whole numbers, so both have the same rounded weights
// The factor 2^20 comes in at a tile's end.
template <bool BF16, int D, int NT>
__global__ void __launch_bounds__(kThreads, Layout<D, NT>::kCtasPerSm) attention4_rows_kernel(const AttentionParams p) {
  using L = Layout<D, NT>;
  constexpr int kSteps = D / 16;                          // of the products with the keys
  constexpr int kTiles = D / 16;                          // of the sums, 16 dimensions each
  constexpr int kChunks = D / 32;                         // 16-byte chunks of a token's codes
  extern __shared__ __align__(128) unsigned char smem[];
  launch_dependents();
  wait_for_prior_grids();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
  Share work;
  if (!share_of<L::kRows, kUnitTokens, kTileUnits>(p, work)) return;
  int i = work.request;
  Request r = request_of(p, i);
  const uint32_t ring = smem_addr(smem) + warp * L::kRing, factors = smem_addr(smem) + L::kTokens + warp * L::kTokenBytes, zeros = factors + kStepTokens * 16;

  while (work.unit < work.end) {
    const int tiles = r.tiles(L::kRows, p), keys = r.key_units(kUnitTokens), span = keys + kTileUnits;
    const int head_tile = static_cast<int>(scaled(1, work.rest, span)), head = head_tile / tiles, tile = head_tile % tiles;
    const int from = static_cast<int>(work.rest - static_cast<unsigned long long>(head_tile) * span);
    const int upto = static_cast<int>(min(static_cast<unsigned long long>(span), from + (work.end - work.unit)));
    const int k0 = max(0, from - kTileUnits), k1 = max(0, upto - kTileUnits);
    const unsigned long long tile_begin = work.unit - from;
    work.unit += upto - from;
    work.rest += upto - from;
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
      // page of granule 32 b + lane (a step has two), -1 where there is none
      auto page_of = [&](int b) {
        const int granule = 32 * b + lane, token = base + (granule >> 1) * kUnitTokens + (granule & 1) * 16;
        const int id = (granule >> 1) < n_steps && token < seen_last ? table[token >> p.page_shift] : -1;
        return static_cast<unsigned>(id) < static_cast<unsigned>(p.pages) ? id : -1;
      };
      // for the batch of 16 steps that is being worked off and the one behind it, and what is read ahead for the next
      int page_0 = page_of(0), page_1 = n_steps > 16 ? page_of(1) : -1, page_ahead = -1;
      auto pages_of = [&](int step, int (&id)[2]) {
        const int batch = (step >> 4) & 1 ? page_1 : page_0;
        id[0] = __shfl_sync(kFull, batch, 2 * step & 31);
        id[1] = __shfl_sync(kFull, batch, (2 * step & 31) + 1);
      };
      // the slot of a page's head and place, for the token `token` in page `id`
      auto row_of = [&](int id, int token) {
        return ((static_cast<long long>(id) * p.kv_heads + head) << p.page_shift) + (token & ((1 << p.page_shift) - 1));
      };
      auto issue = [&](int step) {
        if (step < n_steps) {
          int id[2];
          pages_of(step, id);
          const int token = base + step * kUnitTokens;
          const uint32_t stage = ring + (step % L::kStages) * L::kStage;
          constexpr int kCopies = kStepTokens * kChunks / 64;   // of a granule's keys, and of its values, by the warp
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (id[h] < 0) continue;
            const long long at = row_of(id[h], token + 16 * h) * (D / 2) + lane * 16;
            const int8_t *const k_from = p.k_codes + at, *const v_from = p.v_codes + at;
#pragma unroll
            for (int n = 0; n < kCopies; ++n) {
              const int item = (h * kCopies + n) * 32 + lane;
              const int to = placed<D>(item / kChunks, item % kChunks);
              copy16(stage + to, k_from + n * 512);
              copy16(stage + L::kHalf + to, v_from + n * 512);
            }
          }
          if (lane < 16) {                                 // four tokens' words each: the keys', then the values'
            const int mine = lane & 4 ? id[1] : id[0];
            if (mine >= 0) copy16(stage + L::kWords + lane * 16, (lane < 8 ? p.k_grid : p.v_grid) + row_of(mine, token + 4 * (lane & 7)));
          }
        }
        copies_commit();
      };
      __syncthreads();                                      // the shared memory is free of the last tile's sums
#pragma unroll
      for (int s = 0; s < L::kStages - 1; ++s) issue(s);

      uint32_t q[NT][kSteps][2];
      float factor[NT][2], sum_q[NT][2];                    // of the rows 8 t + 2 c and 8 t + 2 c + 1, whose scores this thread has
      scale_queries<BF16, D, NT>(raw, c, q, factor, sum_q);
      int seen[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) seen[t][h] = r.seen((row0 + min(8 * t + 2 * c + h, rows - 1)) / p.group);
      }

      float acc[NT][kTiles][4], acc_zero[NT][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d) acc[t][d][0] = acc[t][d][1] = acc[t][d][2] = acc[t][d][3] = 0.0f;
        acc_zero[t][0] = acc_zero[t][1] = acc_zero[t][2] = acc_zero[t][3] = 0.0f;
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.0f;
      }

      for (int step = 0; step < n_steps; ++step) {
        copies_wait<L::kStages - 2>();
        __syncwarp();
        issue(step + L::kStages - 1);
        int id[2];
        pages_of(step, id);
        // the batch after the next takes this one's place: its pages are read while this one's last steps are worked off
        if ((step & 15) == 7 && (step | 15) + 17 < n_steps) page_ahead = page_of((step >> 4) + 2);
        if ((step & 15) == 15) {
          if ((step >> 4) & 1) {
            page_1 = page_ahead;
          } else {
            page_0 = page_ahead;
          }
          page_ahead = -1;
        }
        if (id[0] < 0 && id[1] < 0) continue;
        const uint32_t stage = ring + (step % L::kStages) * L::kStage;
        const int token0 = base + step * kUnitTokens;

        // factors of the lane's token: of its scores, their addend (log2 s_v), of the softmax's sum; a token that is not there has weight 0
        {
          const uint32_t k_word = lds32(stage + L::kWords + lane * 4), v_word = lds32(stage + L::kWords + (kStepTokens + lane) * 4);
          const bool here = (lane < 16 ? id[0] : id[1]) >= 0 && token0 + lane < seen_last;
          const float vs = grid_scale(v_word);
          const float ks = grid_is_number(k_word) && grid_is_number(v_word) ? grid_scale(k_word) * p.scale_log2 : NAN;
          asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(factors + lane * 16), "f"(here ? ks : 0.0f), "f"(here ? grid_zero(k_word) : 0.0f),
                       "f"(here ? log2_of_scale(vs) : -INFINITY), "f"(here ? inverse_of_scale(vs) : 0.0f)
                       : "memory");
          const __half z = __float2half_rn(here ? grid_zero(v_word) : 0.0f);
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(zeros + lane * 2), "h"(__half_as_ushort(z)) : "memory");
        }
        __syncwarp();

        // scores of two times 16 tokens and the rows
        float s[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int t = 0; t < NT; ++t) s[u][t][0] = s[u][t][1] = s[u][t][2] = s[u][t][3] = 0.0f;
          uint32_t w0[kChunks], w1[kChunks];                // of the tokens g and g + 8: D / 4 dimensions from c * D / 4 on
          if constexpr (D == 128) {
            const uint4 x0 = lds128(stage + placed<D>(16 * u + g, c)), x1 = lds128(stage + placed<D>(16 * u + g + 8, c));
            w0[0] = x0.x, w0[1] = x0.y, w0[2] = x0.z, w0[3] = x0.w;
            w1[0] = x1.x, w1[1] = x1.y, w1[2] = x1.z, w1[3] = x1.w;
          } else {
            const uint2 x0 = lds64(stage + placed<D>(16 * u + g, c / 2) + 8 * (c % 2)), x1 = lds64(stage + placed<D>(16 * u + g + 8, c / 2) + 8 * (c % 2));
            w0[0] = x0.x, w0[1] = x0.y;
            w1[0] = x1.x, w1[1] = x1.y;
          }
#pragma unroll
          for (int k = 0; k < kChunks; ++k) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t u0 = w0[k] >> (8 * h), u1 = w1[k] >> (8 * h);
              const uint32_t a[4] = {low_nibbles(u0), low_nibbles(u1), high_nibbles(u0), high_nibbles(u1)};
#pragma unroll
              for (int t = 0; t < NT; ++t) mma_16816(s[u][t], a, q[t][2 * k + h][0], q[t][2 * k + h][1]);
            }
          }
        }
        float inverse_v[2][2];
        bool over = false;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float4 f0 = lds128f(factors + (16 * u + g) * 16), f1 = lds128f(factors + (16 * u + g + 8) * 16);
          inverse_v[u][0] = f0.w, inverse_v[u][1] = f1.w;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              s[u][t][h] = __fmaf_rn(__fmaf_rn(f0.y, sum_q[t][h], s[u][t][h]), f0.x * factor[t][h], f0.z);
              s[u][t][2 + h] = __fmaf_rn(__fmaf_rn(f1.y, sum_q[t][h], s[u][t][2 + h]), f1.x * factor[t][h], f1.z);
            }
          }
        }
        if (token0 + kStepTokens > seen_first) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                if (token0 + 16 * u + g >= seen[t][h]) s[u][t][h] = -INFINITY;
                if (token0 + 16 * u + g + 8 >= seen[t][h]) s[u][t][2 + h] = -INFINITY;
              }
            }
          }
        }
        float top[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            top[t][h] = fmaxf(fmaxf(s[0][t][h], s[0][t][2 + h]), fmaxf(s[1][t][h], s[1][t][2 + h]));
            over = over || top[t][h] > m[t][h] + 8.0f;
          }
        }
        // m is a reference, not the maximum: it follows only when a score is more than 2^8 above it (a weight stays below 2^9 in binary16)
        if (__any_sync(kFull, over)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float by[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float now = fmaxf(m[t][h], column_max(top[t][h]));
              by[h] = m[t][h] == -INFINITY ? 0.0f : exp2_fast(m[t][h] - now);
              m[t][h] = now;
              l[t][h] *= by[h];
              acc_zero[t][h] *= by[h];
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
        uint32_t w[2][NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float ref0 = m[t][0] == -INFINITY ? 0.0f : m[t][0], ref1 = m[t][1] == -INFINITY ? 0.0f : m[t][1];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float x0 = exp2_fast(s[u][t][0] - ref0), x1 = exp2_fast(s[u][t][1] - ref1), x2 = exp2_fast(s[u][t][2] - ref0), x3 = exp2_fast(s[u][t][3] - ref1);
            l[t][0] = __fmaf_rn(x0, inverse_v[u][0], __fmaf_rn(x2, inverse_v[u][1], l[t][0]));
            l[t][1] = __fmaf_rn(x1, inverse_v[u][0], __fmaf_rn(x3, inverse_v[u][1], l[t][1]));
            w[u][t][0] = transposed(pack_half2(x0, x1));
            w[u][t][1] = transposed(pack_half2(x2, x3));
          }
        }

        // values: thread (g, c) has the dimensions g * D / 8 ... of the tokens 2c, 2c + 1, 2c + 8, 2c + 9
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          uint32_t v[4][D / 64];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int token = 16 * u + 2 * c + (t & 1) + 8 * (t >> 1);
            if constexpr (D == 128) {
              const uint2 x = lds64(stage + L::kHalf + placed<D>(token, g / 2) + 8 * (g % 2));
              v[t][0] = x.x, v[t][1] = x.y;
            } else {
              v[t][0] = lds32(stage + L::kHalf + placed<D>(token, g / 4) + 4 * (g % 4));
            }
          }
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {          // four codes of a token beside four of its neighbour
              const uint32_t x = __byte_perm(v[0][k], v[1][k], half ? 0x7632 : 0x5410), y = __byte_perm(v[2][k], v[3][k], half ? 0x7632 : 0x5410);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t u0 = x >> (8 * h), u1 = y >> (8 * h);
                const uint32_t a[4] = {low_nibbles(u0), high_nibbles(u0), low_nibbles(u1), high_nibbles(u1)};
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_16816(acc[t][4 * k + 2 * half + h], a, w[u][t][0], w[u][t][1]);
              }
            }
          }
          const uint32_t z0 = lds32(zeros + (16 * u + 2 * c) * 2), z1 = lds32(zeros + (16 * u + 2 * c + 8) * 2);
          const uint32_t a[4] = {g == 0 ? z0 : 0u, 0u, g == 0 ? z1 : 0u, 0u};
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_16816(acc_zero[t], a, w[u][t][0], w[u][t][1]);
        }
      }

      // codes' sums and zero-points' sum in one measure: the latter are with the threads of g = 0
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float zero0 = __shfl_sync(kFull, acc_zero[t][0], c), zero1 = __shfl_sync(kFull, acc_zero[t][1], c);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
          acc[t][d][0] = __fmaf_rn(acc[t][d][0], 1048576.0f, zero0);
          acc[t][d][1] = __fmaf_rn(acc[t][d][1], 1048576.0f, zero1);
          acc[t][d][2] = __fmaf_rn(acc[t][d][2], 1048576.0f, zero0);
          acc[t][d][3] = __fmaf_rn(acc[t][d][3], 1048576.0f, zero1);
        }
      }
      finish_tile<BF16, D, NT>(p, work, r, head, row0, rows, k0 > 0 || k1 < keys, tile_begin + kTileUnits, tile_begin + span - 1, smem, m, l, acc);
    }
    if (work.unit < work.end && work.rest == r.units(L::kRows, kUnitTokens, kTileUnits, p)) {
      do {
        r = request_of(p, ++i);
      } while (r.rows == 0 && i + 1 < p.requests);
      if (r.rows == 0) break;                             // not reached while units are left
      work.rest = 0;
    }
  }
}

template <bool BF16, int D, int NT>
cudaError_t launch(const AttentionParams& p, int sms, cudaStream_t stream) {
  using L = Layout<D, NT>;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_shared(attention4_rows_kernel<BF16, D, NT>, L::kBytes, done);
  if (e != cudaSuccess) return e;
  return launch_overlapped(attention4_rows_kernel<BF16, D, NT>, sms * L::kCtasPerSm, kThreads, static_cast<size_t>(L::kBytes), stream, p);
}

template <bool BF16, int D>
cudaError_t launch(const AttentionParams& p, int sms, cudaStream_t stream) {
  return static_cast<long long>(p.max_query) * p.group <= 8 ? launch<BF16, D, 1>(p, sms, stream) : launch<BF16, D, 2>(p, sms, stream);
}

}  // namespace

cudaError_t launch_attention4_rows(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream) {
  if (head_dim == 128) return bf16 ? launch<true, 128>(p, sms, stream) : launch<false, 128>(p, sms, stream);
  return bf16 ? launch<true, 64>(p, sms, stream) : launch<false, 64>(p, sms, stream);
}

}  // namespace tsq
