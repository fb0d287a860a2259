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
constexpr int kTileUnits = 2;                // what beginning and ending a tile costs, in units

constexpr uint32_t kNoToken = 0xff80u;       // the word of a token without a page: no scale is negative

__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}

__device__ __forceinline__ void lds2x64(uint64_t& a, uint64_t& b, uint32_t at) { asm volatile("ld.shared.v2.u64 {%0,%1}, [%2];" : "=l"(a), "=l"(b) : "r"(at)); }
// The first of a row of products.
__device__ __forceinline__ void mma_16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}

// Where the 16-byte chunk `c` of token row `t` lies in a stage: chunks change places within their 128 bytes, so that the eight chunks that lanes read at once of every second
// row lie in different banks.
template <int D>
__device__ __forceinline__ int placed(int t, int c) {
  const int at = t * (D / 32) + c;
  return (at ^ (D == 128 ? ((at >> 3) & 3) << 1 : ((at >> 3) & 1) << 1)) << 4;
}

// The queries as the products with nibbles take them, brought to binary16 by a power of two per row.  Of eight dimensions the pairs (0, 4), (1, 5), (2, 6), (3, 7) go together;
// odd ones meet codes that count sixteen times.  factor, sum: of the rows 8 t + 2 c and 8 t + 2 c + 1, what turns sums of products into <q, code>, and the row's sum in their measure.
template <bool BF16, int D, int NT>
__device__ __forceinline__ void scale_queries(const uint4 (&raw)[NT][D / 32], int c, uint32_t (&q)[NT][D / 16][2], uint64_t (&factor)[NT], uint64_t (&sum)[NT]) {
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
    const float power = row_power<126>(Elem<BF16>::pattern_f32(top), inverse);  // a sixteenth of the least numbers is to be one, too
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t u = w[4 * k + h], v = w[4 * k + 2 + h];
        const float u0 = Elem<BF16>::lo_f32(u) * power, v0 = Elem<BF16>::lo_f32(v) * power, u1 = Elem<BF16>::hi_f32(u) * power, v1 = Elem<BF16>::hi_f32(v) * power;
        q[t][2 * k + h][0] = pack_half2(u0, v0);
        q[t][2 * k + h][1] = pack_half2(u1 * 0.0625f, v1 * 0.0625f);
        all += (u0 + v0) + (u1 + v1);
      }
    }
    all += __shfl_xor_sync(kFull, all, 1);
    all += __shfl_xor_sync(kFull, all, 2);
    all *= 4.76837158203125e-7f;                           // 2^-21
    inverse *= 2097152.0f;                                 // the 2^21 that a code lacks
    factor[t] = pack2f(__shfl_sync(kFull, inverse, 8 * c), __shfl_sync(kFull, inverse, 8 * c + 4));  // of the threads with g = 2 c and 2 c + 1
    sum[t] = pack2f(__shfl_sync(kFull, all, 8 * c), __shfl_sync(kFull, all, 8 * c + 4));
  }
}

// Tiles of 8 query rows (NT = 1) or 16 (NT = 2).
template <int D, int NT>
struct Layout {
  static constexpr int kRows = 8 * NT;
  // heads of 128, 8 rows: 4 CTAs of 128 registers 70.5 us for 64 requests, 3 of 168 68.2, 2 of 255 73; 131072 tokens 46.0, 40.5, 42.6.  16 rows: 3 CTAs 58.9 us for 16 requests of 8000 tokens, 2
  // (nothing spilled) 50.7; heads of 64 3 CTAs 35.2 (20 bytes spilled), 2 35.6
  static constexpr int kCtasPerSm = D == 64 ? (NT == 1 ? 4 : 3) : NT == 1 ? 3 : 2;
  static constexpr int kStages = 3;                      // of a warp's ring
  static constexpr int kHalf = kStepTokens * D / 2;      // bytes of a stage's keys, and of its values
  static constexpr int kWords = 2 * kHalf;               // behind them: the keys' words, the values'
  static constexpr int kStage = kWords + 2 * kStepTokens * 4;
  static constexpr int kRing = kStages * kStage;         // of a warp
  static constexpr int kMerge = RowsSums<D, NT>::kBytes;
  static constexpr int kTokens = kWarps * kRing > kMerge ? kWarps * kRing : kMerge;  // a step's factors for each warp: four numbers a token, each twice, the values' zero-points in binary16, as many zeros
  static constexpr int kTokenBytes = kStepTokens * 36;
  static constexpr int kBytes = kTokens + kWarps * kTokenBytes;
};

// As over the 8-bit cache (tsq_cache_rows.cu): units of neighbouring tokens of one (request, key head, tile of query rows), the same number for every CTA; the four warps have 32
// tokens of a unit each, a ring of stages and sums of their own; codes are the 16-row operand of both products.  What 4 bits change:
//
// A nibble alone in the right bits of a 16-bit field is a binary16 number (to_linear_bits).  So a word becomes four operand registers by two shifts and four masks: (0, 4) and (1, 5) of its
// eight codes, then (2, 6) and (3, 7).  What that leaves is put right outside of the products:
//   score  = s_k (sum q c + z_k sum q)          by two operations per score, the keys' scale and zero-point by token
//   out    = (sum w c + sum w z_v) / sum p      w = p s_v rounded to binary16, as over the 8-bit cache: 2^(score + log2 s_v - m), relative to the row's largest;
//                                               the second sum is one more product, whose operand is the zero-points, whole numbers, so both have the same rounded weights
// The factors 2^21 and 2^17 come in at a tile's end.
//
// Bound by the ALU pipe (half a pass per clock; 5.5 of its operations for 8 codes) and HBM together where the cache is long: 5.6 TB/s from 16000 tokens a request on (64 requests), 4.3 TB/s with what it
// costs to begin and to end for 64 requests of 500 to 8000 tokens (297 MB, 68 to 73 us); by the chain lengths -> table -> codes -> sums where it is short (one of 1001 tokens: 8.5 us).  A step has 32
// tokens, twice as many as over the 8-bit cache: what it costs besides its codes is shared by as many bytes.  Tried and not kept: products of e4m3 with the queries in parts (these instructions come
// out as conversions and products in binary16: 83 us); the next step's scores formed during this one's sums (70.8); the next tile's first codes fetched before a tile's end (68.3, and 28.4 -> 29.5 for many
// short tiles); shares by how early a CTA is launched (70.5).
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
  const uint32_t ring = smem_addr(smem) + warp * L::kRing, factors = smem_addr(smem) + L::kTokens + warp * L::kTokenBytes, zeros = factors + kStepTokens * 32;
  // where the lane's parts lie in a stage (placed), for tokens in front of which a whole number of eight lies: rows of eight are kHalf / 4 apart
  constexpr int kEight = L::kHalf / 4;
  const uint32_t copy_to = placed<D>(lane / kChunks, lane % kChunks);
  const uint32_t k_at = D == 128 ? placed<D>(g, c) : placed<D>(g, c / 2) + 8 * (c % 2);
  const uint32_t v_at = L::kHalf + (D == 128 ? placed<D>(2 * c, g / 2) + 8 * (g % 2) : placed<D>(2 * c, g / 4) + 4 * (g % 4));
  constexpr uint32_t kNeighbour = D == 128 ? 64 : 32;      // token 2 c + 1: that bit of the address the other way round
  // zero-points are one row of their operand; the other rows' threads read zeros behind them
  const uint32_t z_at = zeros + (g == 0 ? 4 * c : 2 * kStepTokens);
  if (lane < 16) asm volatile("st.shared.u32 [%0], %1;" ::"r"(zeros + 2 * kStepTokens + 4 * lane), "r"(0u) : "memory");

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
      // A step's places in its pages are those of every other step.  Addresses in page 0; what a page has of all heads lies `page_rows` rows behind.
      const int place = base & ((1 << p.page_shift) - 1);
      const bool one_page = p.page_shift > 4;               // a step's second granule lies behind the first
      const long long row = (static_cast<long long>(head) << p.page_shift) + place;
      const uint32_t page_rows = static_cast<uint32_t>(p.kv_heads) << p.page_shift, page_bytes = page_rows * (D / 2);
      const int8_t *const k_from = p.k_codes + row * (D / 2) + lane * 16, *const v_from = p.v_codes + row * (D / 2) + lane * 16;
      // lanes 0 .. 15: four tokens' words each, the keys', then the values'
      const uint32_t* const words_from = (lane & 8 ? p.v_grid : p.k_grid) + row + (lane & 3) * 4 + (lane & 4 && one_page ? 16 : 0);
      uint32_t stage_in = ring;
      auto issue = [&](int step) {
        if (step < n_steps) {
          const int batch = (step >> 4) & 1 ? page_1 : page_0;
          const int id0 = __shfl_sync(kFull, batch, 2 * step & 31), id1 = __shfl_sync(kFull, batch, (2 * step & 31) + 1);
          constexpr int kCopies = kStepTokens * kChunks / 64;   // of a granule's keys, and of its values, by the warp
          const auto copy_granules = [&](int id, int first, int n_granules) {
            const int8_t* const k_page = k_from + static_cast<unsigned long long>(static_cast<uint32_t>(id)) * page_bytes;
            const int8_t* const v_page = v_from + static_cast<unsigned long long>(static_cast<uint32_t>(id)) * page_bytes;
#pragma unroll
            for (int n = 0; n < n_granules * kCopies; ++n) {
              const uint32_t to = stage_in + copy_to + (first * kCopies + n) * 512;
              copy16(to, k_page + n * 512);
              copy16(to + L::kHalf, v_page + n * 512);
            }
          };
          if (one_page && (id0 | id1) >= 0) {               // the second granule of the last step may have no token
            copy_granules(id0, 0, 2);
          } else {                                          // one_page: the second one is then not there
            if (id0 >= 0) copy_granules(id0, 0, 1);
            if (id1 >= 0) copy_granules(id1, 1, 1);
          }
          const int mine = lane & 4 ? id1 : id0;
          if (lane < 16) {
            const uint32_t to = stage_in + L::kWords + lane * 16;
            if (mine >= 0) {
              copy16(to, words_from + static_cast<unsigned long long>(static_cast<uint32_t>(mine)) * page_rows);
            } else {
              asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(kNoToken) : "memory");
            }
          }
        }
        copies_commit();
        stage_in = stage_in + L::kStage == ring + L::kRing ? ring : stage_in + L::kStage;
      };
      __syncthreads();                                      // the shared memory is free of the last tile's sums
#pragma unroll
      for (int s = 0; s < L::kStages - 1; ++s) issue(s);

      uint32_t q[NT][kSteps][2];
      uint64_t factor[NT], sum_q[NT];                       // of the rows 8 t + 2 c and 8 t + 2 c + 1, whose scores this thread has
      scale_queries<BF16, D, NT>(raw, c, q, factor, sum_q);
      int seen[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) seen[t][h] = r.seen((row0 + min(8 * t + 2 * c + h, rows - 1)) / p.group);
      }

      float acc[NT][kTiles][4], acc_zero[NT][4];
      float m[NT][2], limit[NT][2];
      uint64_t l[NT], less[NT];                             // sums; the references negated, 0 as long as there is none
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d) acc[t][d][0] = acc[t][d][1] = acc[t][d][2] = acc[t][d][3] = 0.0f;
        acc_zero[t][0] = acc_zero[t][1] = acc_zero[t][2] = acc_zero[t][3] = 0.0f;
        m[t][0] = m[t][1] = limit[t][0] = limit[t][1] = -INFINITY;
        l[t] = less[t] = 0ull;
      }

      uint32_t stage_out = ring;
      for (int step = 0; step < n_steps; ++step) {
        copies_wait<L::kStages - 2>();
        __syncwarp();
        issue(step + L::kStages - 1);
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
        const uint32_t stage = stage_out;
        stage_out = stage + L::kStage == ring + L::kRing ? ring : stage + L::kStage;
        const int token0 = base + step * kUnitTokens;

        // factors of the lane's token: of its scores, their addend (log2 s_v), of the softmax's sum; a token that is not there has weight 0
        {
          uint32_t k_word = lds32(stage + L::kWords + lane * 4), v_word = lds32(stage + L::kWords + (kStepTokens + lane) * 4);
          const bool here = v_word != kNoToken && token0 + lane < seen_last;
          k_word = here ? k_word : 0u;
          v_word = here ? v_word : 0u;
          const float ks = grid_scale(k_word), vs = grid_scale(v_word), least = fmaxf(vs, kLeastScale), kz = grid_zero(k_word);
          const float by = __fmaf_rn(ks, p.scale_log2, __fmaf_rn(ks, 0.0f, vs * 0.0f));  // NaN where one of the scales is not finite
          const float a = here ? log2_approx(least) : -INFINITY, inverse = reciprocal(least);
          // each twice, for the products of pairs of rows
          asm volatile("st.shared.v4.f32 [%0], {%1,%1,%2,%2};" ::"r"(factors + lane * 32), "f"(by), "f"(kz) : "memory");
          asm volatile("st.shared.v4.f32 [%0], {%1,%1,%2,%2};" ::"r"(factors + lane * 32 + 16), "f"(a), "f"(inverse) : "memory");
          const __half z = __float2half_rn(grid_zero(v_word));
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(zeros + lane * 2), "h"(__half_as_ushort(z)) : "memory");
        }
        __syncwarp();

        // scores of two times 16 tokens and the rows
        float s[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          uint32_t w0[kChunks], w1[kChunks];                // of the tokens g and g + 8: D / 4 dimensions from c * D / 4 on
          if constexpr (D == 128) {
            const uint4 x0 = lds128(stage + k_at + 2 * u * kEight), x1 = lds128(stage + k_at + (2 * u + 1) * kEight);
            w0[0] = x0.x, w0[1] = x0.y, w0[2] = x0.z, w0[3] = x0.w;
            w1[0] = x1.x, w1[1] = x1.y, w1[2] = x1.z, w1[3] = x1.w;
          } else {
            const uint2 x0 = lds64(stage + k_at + 2 * u * kEight), x1 = lds64(stage + k_at + (2 * u + 1) * kEight);
            w0[0] = x0.x, w0[1] = x0.y;
            w1[0] = x1.x, w1[1] = x1.y;
          }
#pragma unroll
          for (int k = 0; k < kChunks; ++k) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t u0 = to_linear_bits(w0[k], h != 0), u1 = to_linear_bits(w1[k], h != 0);
              const uint32_t a[4] = {low_nibbles(u0), low_nibbles(u1), high_nibbles(u0), high_nibbles(u1)};
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                if (k + h == 0) {
                  mma_16816_first(s[u][t], a, q[t][0][0], q[t][0][1]);
                } else {
                  mma_16816(s[u][t], a, q[t][2 * k + h][0], q[t][2 * k + h][1]);
                }
              }
            }
          }
        }
        uint64_t inverse_v[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {                     // tokens g and g + 8
            uint64_t by, kz, a;
            lds2x64(by, kz, factors + (16 * u + 8 * e + g) * 32);
            lds2x64(a, inverse_v[u][e], factors + (16 * u + 8 * e + g) * 32 + 16);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint64_t x = fma2(fma2(kz, sum_q[t], pack2f(s[u][t][2 * e], s[u][t][2 * e + 1])), mul2(by, factor[t]), a);
              unpack2f(x, s[u][t][2 * e], s[u][t][2 * e + 1]);
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
        bool over = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            top[t][h] = fmaxf(fmaxf(s[0][t][h], s[0][t][2 + h]), fmaxf(s[1][t][h], s[1][t][2 + h]));
            over = over || top[t][h] > limit[t][h];
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
              limit[t][h] = follow_above(now);
              acc_zero[t][h] *= by[h];
            }
            l[t] = mul2(l[t], pack2f(by[0], by[1]));
            less[t] = pack2f(m[t][0] == -INFINITY ? 0.0f : -m[t][0], m[t][1] == -INFINITY ? 0.0f : -m[t][1]);
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
#pragma unroll
          for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x0, x1;
              unpack2f(add2(pack2f(s[u][t][2 * e], s[u][t][2 * e + 1]), less[t]), x0, x1);
              x0 = exp2_fast(x0);
              x1 = exp2_fast(x1);
              l[t] = fma2(pack2f(x0, x1), inverse_v[u][e], l[t]);
              w[u][t][e] = transposed(pack_half2(x0, x1));
            }
          }
        }

        // values: thread (g, c) has the dimensions g * D / 8 ... of the tokens 2c, 2c + 1, 2c + 8, 2c + 9
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          uint32_t v[4][D / 64];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t at = (stage + (t & 1 ? v_at ^ kNeighbour : v_at)) + (2 * u + (t >> 1)) * kEight;
            if constexpr (D == 128) {
              const uint2 x = lds64(at);
              v[t][0] = x.x, v[t][1] = x.y;
            } else {
              v[t][0] = lds32(at);
            }
          }
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {          // four codes of a token beside four of its neighbour
              const uint32_t x = __byte_perm(v[0][k], v[1][k], half ? 0x7632 : 0x5410), y = __byte_perm(v[2][k], v[3][k], half ? 0x7632 : 0x5410);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t u0 = to_linear_bits(x, h != 0), u1 = to_linear_bits(y, h != 0);
                const uint32_t a[4] = {low_nibbles(u0), high_nibbles(u0), low_nibbles(u1), high_nibbles(u1)};
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_16816(acc[t][4 * k + 2 * half + h], a, w[u][t][0], w[u][t][1]);
              }
            }
          }
          const uint32_t a[4] = {lds32(z_at + 32 * u), 0u, lds32(z_at + 32 * u + 16), 0u};
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_16816(acc_zero[t], a, w[u][t][0], w[u][t][1]);
        }
      }

      float sums[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) unpack2f(l[t], sums[t][0], sums[t][1]);
      // codes' sums and zero-points' sum in one measure: the latter are with the threads of g = 0
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float zero0 = __shfl_sync(kFull, acc_zero[t][0], c), zero1 = __shfl_sync(kFull, acc_zero[t][1], c);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
          acc[t][d][0] = __fmaf_rn(acc[t][d][0], 2097152.0f, zero0);
          acc[t][d][1] = __fmaf_rn(acc[t][d][1], 2097152.0f, zero1);
          acc[t][d][2] = __fmaf_rn(acc[t][d][2], 131072.0f, zero0);
          acc[t][d][3] = __fmaf_rn(acc[t][d][3], 131072.0f, zero1);
        }
      }
      finish_tile<BF16, D, NT>(p, work, r, head, row0, rows, k0 > 0 || k1 < keys, tile_begin + kTileUnits, tile_begin + span - 1, smem, m, sums, acc);
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
