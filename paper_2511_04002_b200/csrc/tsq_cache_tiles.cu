// Attention over the paged 8-bit cache for many query rows per request (prompts, chunks of prompts), on the tensor cores' asynchronous products.

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_device.cuh"
#include "tsq_internal.h"

namespace tsq {
namespace {

constexpr int kKeys = 128;                   // tokens of a step
constexpr int kGranules = kKeys / 16;        // parts of a step that lie within one page
constexpr int kThreads = 5 * 128;            // two softmax warpgroups, two that widen codes, one whose first two warps issue the products
// Registers: 96 a thread at launch, dealt out again among the five: 2 * 136 + 2 * 80 + 48 = 5 * 96.
constexpr int kSoftmaxRegs = 136, kWidenRegs = 80, kProductRegs = 48, kLaunchRegs = 96;
constexpr int kTileSteps = 4;                // what beginning and ending a tile costs, in steps
// Most parts of a tile, on the average: adding a part up takes 1.7 us, a step 2.3 us (one tile of 235 steps in 148 parts 300 us, in 16 80 us).
constexpr unsigned long long kMostParts = 16;
constexpr int kMeta = 4;                     // steps whose scales are kept
constexpr uint32_t kPolls = 1u << 20;        // of a wait inside the CTA: tens of milliseconds at least, where a sound one takes microseconds

// ---- barriers, tensor memory, products -----------------------------------------------------------

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
// One arrival for the warp, behind what its threads have done (and fenced, where another proxy is to see it).
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) asm volatile("{\n\t.reg .b64 s;\n\tmbarrier.arrive.shared::cta.b64 s, [%0];\n\t}" ::"r"(bar) : "memory");
}
// Whether the phase of that parity has ended; false after kPolls polls.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t n = 0; n < kPolls; ++n) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    if (done) return true;
  }
  return false;
}

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
// The end of a role: back to the launch's registers, so that the code behind the roles may use any of those, whichever role a warp comes from.  (Behind roles of
// different counts nothing keeps a value out of the registers that the smallest role has given away.)  The warps of a warpgroup meet between two setmaxnreg.
template <int N>
__device__ __forceinline__ void regs_back(int group, bool failed, uint32_t* s_failed) {
  if (failed) *s_failed = 1u;
  asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory");
  if constexpr (N > kLaunchRegs) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLaunchRegs));
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kLaunchRegs));
  }
}
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void tm_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_commit(uint32_t leader, uint32_t bar) {
  asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.u32 e, %1, 0;\n\t@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
}

#define TSQ_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define TSQ_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of the warp's 32 lanes
__device__ __forceinline__ void tm_load32(uint32_t (&v)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, "
      "[%32];"
      : TSQ_R8(v, 0), TSQ_R8(v, 8), TSQ_R8(v, 16), TSQ_R8(v, 24)
      : "r"(at));
}
// What is computed from loaded registers has to stay behind the wait: they pass through it.
#define TSQ_RW8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
__device__ __forceinline__ void tm_wait_ld(uint32_t (&v)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : TSQ_RW8(v, 0), TSQ_RW8(v, 8)::"memory"); }
__device__ __forceinline__ void tm_wait_ld(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : TSQ_RW8(v, 0), TSQ_RW8(v, 8)::"memory");
  asm volatile("" : TSQ_RW8(v, 16), TSQ_RW8(v, 24)::"memory");
}
__device__ __forceinline__ void tm_load16(uint32_t (&v)[16], uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : TSQ_R8(v, 0), TSQ_R8(v, 8) : "r"(at));
}
__device__ __forceinline__ void tm_store32(uint32_t at, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
      "%32};" ::"r"(at),
      TSQ_W8(v, 0), TSQ_W8(v, 8), TSQ_W8(v, 16), TSQ_W8(v, 24)
      : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), TSQ_W8(v, 0), TSQ_W8(v, 8) : "memory");
}
__device__ __forceinline__ float4 shared_float4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
  return v;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Largest score of 32 keys (two granules, whose scales lie at `scales`; a granule has one factor that is not negative) in the form that the weights' exponent has; with MASK only the first `left` count.
template <bool MASK>
__device__ __forceinline__ float top_score(const uint32_t (&scores)[32], uint32_t scales, float by_scale, int left) {
  uint32_t s[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) s[e] = scores[e];
  if constexpr (MASK) {
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = e < left ? s[e] : 0xff800000u;
  }
  float most = -INFINITY;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const uint32_t* const x = s + 16 * g;
    float t0 = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2])), t1 = max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5]));
    t0 = max3(t0, __uint_as_float(x[6]), __uint_as_float(x[7]));
    t1 = max3(t1, __uint_as_float(x[8]), __uint_as_float(x[9]));
    t0 = max3(t0, __uint_as_float(x[10]), __uint_as_float(x[11]));
    t1 = max3(t1, __uint_as_float(x[12]), __uint_as_float(x[13]));
    t0 = max3(t0, __uint_as_float(x[14]), __uint_as_float(x[15]));
    const float raw = fmaxf(t0, t1);
    const float4 f = shared_float4(scales + 16 * g);       // score factor, log2 and inverse of the values' scale
    const float v = __fmaf_rn(raw, f.x * by_scale, f.y);
    most = fmaxf(most, raw == -INFINITY ? raw : v);
  }
  return most;
}
// References up to this take part in the product's addend, f.y - m: that is off by up to 2^-5 there.  Beyond, it could be off by more than any weight may be in binary16
// (from 2^27 on by 8 and more), so a score is formed as the reference was and the reference subtracted from it: the largest key's difference is 0 whatever m is.
constexpr float kNearReference = 1048576.0f;  // 2^20

// Weights of 32 keys in binary16, two to a word; their sum over the values' scale is added to l.  most: the largest sum of a granule's weights, and so no less than any weight.
// FAR: references of any size; one that is near gives the same bits as without.
template <bool MASK, bool FAR>
__device__ __forceinline__ void weights_of_32(const uint32_t (&s)[32], uint32_t* w, uint32_t scales, float by_scale, float m, float& l, float& most, int left) {
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float4 f = shared_float4(scales + 16 * g);
    const bool far = FAR && fabsf(m) >= kNearReference;
    const float a = f.x * by_scale, b = far ? f.y : f.y - m, less = far ? m : 0.0f;
    const uint64_t a2 = pack2f(a, a), b2 = pack2f(b, b);
    uint64_t sum = 0ull;                                   // of even and of odd keys
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      float x0, x1;
      unpack2f(fma2(pack2u(s[16 * g + e], s[16 * g + e + 1]), a2, b2), x0, x1);
      if constexpr (FAR) {
        x0 -= less;
        x1 -= less;
      }
      if constexpr (MASK) {
        x0 = 16 * g + e < left ? x0 : -INFINITY;
        x1 = 16 * g + e + 1 < left ? x1 : -INFINITY;
      }
      x0 = exp2_fast(x0);
      x1 = exp2_fast(x1);
      sum = add2(sum, pack2f(x0, x1));
      w[8 * g + e / 2] = pack_half2(x0, x1);
    }
    float even, odd;
    unpack2f(sum, even, odd);
    most = fmaxf(most, even + odd);
    l = __fmaf_rn(even + odd, f.z, l);
  }
}
template <bool MASK, bool FAR>
__device__ __forceinline__ float weights_of(const uint32_t (&a)[32], const uint32_t (&b)[32], uint32_t (&w)[32], uint32_t scales, float by_scale, float m, float& most,
                                            int left) {
  float sum = 0.0f;
  most = 0.0f;
  weights_of_32<MASK, FAR>(a, w, scales, by_scale, m, sum, most, left);
  weights_of_32<MASK, FAR>(b, w + 16, scales + 32, by_scale, m, sum, most, left - 32);
  return sum;
}

// 32 bytes at once where they are a sector, which neighbouring threads' rows do not share.
__device__ __forceinline__ void load_sector(uint4& a, uint4& b, const void* at) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
               : "l"(at));
}
__device__ __forceinline__ void store_sector(void* at, const uint32_t (&w)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), TSQ_W8(w, 0) : "memory");
  } else {
    static_cast<uint4*>(at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    static_cast<uint4*>(at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// Shared-memory descriptors of 128-byte swizzled operands: rows of 128 bytes, eight rows to a 1024-byte atom.
// K-major (queries, keys): atoms follow one another down the rows.  MN-major (values: a row is a token, its 64 dimensions contiguous): atoms follow
// one another along the tokens, the second 64 dimensions lie kHalf bytes behind.
constexpr int kHalf = 128 * 128;             // 128 rows of 64 binary16 numbers
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading, uint32_t stride) {
  return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | static_cast<uint64_t>(leading >> 4) << 16 | static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor: binary32 sums, binary16 operands, 128 rows.
__host__ __device__ constexpr uint32_t product_of(int columns, bool b_mn_major) {
  return 1u << 4 | (b_mn_major ? 1u << 16 : 0u) | static_cast<uint32_t>(columns / 8) << 17 | (128u / 16u) << 24;
}
// The whole warp comes here and `leader` is set in one thread of it: a guard on the instruction instead of a branch around it leaves the operands' arithmetic to
// the warp's uniform registers, from which the instruction takes them.
__device__ __forceinline__ void product_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 e, %5, 0;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
      "r"(what), "r"(static_cast<uint32_t>(add)), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 e, %5, 0;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
      "r"(what), "r"(static_cast<uint32_t>(add)), "r"(leader)
      : "memory");
}
__device__ __forceinline__ uint32_t elected() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(kFull, v, 0); }

// ---- work ----------------------------------------------------------------------------------------

// Steps of the tile of 256 rows that begins at row0: by the keys its last row sees, one at least.
__device__ __forceinline__ int steps_of(const Request& r, uint32_t rows, uint32_t row0, const AttentionParams& p) {
  const int seen = r.seen(static_cast<int>((min(rows, row0 + kTilesRows) - 1u) / static_cast<uint32_t>(p.group)));
  return seen > 0 ? (seen - 1) / kKeys + 1 : 1;
}

// Where a CTA is in its share of the work.  Order: request, key head, tile of rows, step; in front of a tile's steps lie kTileSteps units that stand for
// what beginning and ending it costs.
struct Place {
  int request, head, tile;
  Request r;
  uint32_t rows;                  // rows of the request times the group, below 2^31 (tsq_cache_attention)
  int steps;                      // of the tile
  int from, upto;                 // units that the CTA takes of it,
  int k0, k1;                     // and steps
  int before;                     // steps that the CTA has had before
  unsigned long long unit, end;   // the first unit; where the CTA's share ends

  __device__ __forceinline__ void take(const AttentionParams& p) {
    steps = steps_of(r, rows, static_cast<uint32_t>(tile) * kTilesRows, p);
    upto = static_cast<int>(min(static_cast<unsigned long long>(steps + kTileSteps), from + (end - unit)));
    k0 = max(0, from - kTileSteps);
    k1 = max(0, upto - kTileSteps);
  }
  // the next tile of which the CTA has steps
  __device__ __forceinline__ bool next(const AttentionParams& p) {
    do {
      unit += upto - from;
      before += k1 - k0;
      if (unit >= end) return false;
      from = 0;
      if (static_cast<uint32_t>(++tile) * kTilesRows >= rows) {
        tile = 0;
        if (++head == p.kv_heads) {
          head = 0;
          do {
            if (++request >= p.requests) return false;
            r = request_of(p, request);
          } while (r.rows == 0);
          rows = static_cast<uint32_t>(r.rows) * static_cast<uint32_t>(p.group);
        }
      }
      take(p);
    } while (k1 == k0);
    return true;
  }
  // steps of the half of the tile (128 rows) that group t has: as far as its last row sees, 0 where it has no row
  __device__ __forceinline__ int limit(int t, const AttentionParams& p) const {
    const uint32_t row0 = static_cast<uint32_t>(tile) * kTilesRows + 128u * t;
    if (row0 >= rows) return 0;
    const int seen = r.seen(static_cast<int>((min(rows, row0 + 128u) - 1u) / static_cast<uint32_t>(p.group)));
    return min(k1, seen > 0 ? (seen - 1) / kKeys + 1 : 1);
  }
};

template <int D>
struct Shared {
  static constexpr int kHalves = D / 64;
  static constexpr int kOperand = kHalves * kHalf;        // 128 rows of D binary16 numbers
  static constexpr int kQ = 0, kK = 2 * kOperand, kV = 4 * kOperand;
  static constexpr int kScales = 6 * kOperand;
  static constexpr int kBars = kScales + kMeta * kGranules * 16;
  static constexpr int kBytes = kBars + 256;
};
// Barriers: buffers of keys and values; a half step's scores, weights and sums, by group and half; a tile's queries, by group; the end of a group's products.
enum Bar { kKFull = 0, kKFree = 2, kVFull = 4, kVFree = 6, kSFull = 8, kPReady = 12, kODone = 16, kQFull = 20, kEnd = 22, kBarCount = 24 };
__host__ __device__ constexpr uint32_t arrivals_of(int bar) {  // a group's warps, or one for the products of each group
  return bar < kKFree || (bar >= kVFull && bar < kVFree) || (bar >= kPReady && bar < kODone) || (bar >= kQFull && bar < kEnd) ? 4u : bar >= kKFree && bar < kSFull ? 2u : 1u;
}

// A CTA's two groups of 128 threads have 128 query rows each, a thread a row; a tile is the 256 rows of one (request, key head) that follow one another, the group's query
// heads of a token side by side, so that widened codes serve both groups and all heads.  Per step of 128 tokens:
//   widening groups one for the keys, one for the values: codes from global memory (a step ahead in registers) to binary16 (exact) in shared memory, two buffers each
//   product warps   one for each group: S = Q K^T into tensor memory, then O += P V with P from tensor memory
//   softmax groups  S out of tensor memory, w = 2^(S * scale + log2 s_v - m) to binary16 in S's place, sums in binary32
// Scores come in halves of 64 keys, each with its place in tensor memory: while a group works on one, its products fill the other, and the other group's run besides.
// m is a reference that follows the row's maximum only when weights come out above 2^12: then the half is done again and O is scaled in tensor memory.  Every CTA takes the
// same number of steps whatever the requests' lengths are; tiles that several CTAs have a part of are added up through the workspace by the one that comes last, in the
// order of the steps.
// Bound by the chain scores -> weights -> sums -> scores of each group: about 4400 clocks a step where the products take 2050 and the exponentials, 16 per SM and clock, as many.
// 8192 tokens, 32 query heads on 8 key heads: 600 to 634 us, 865 to 910 TFLOP/s (bf16 or fp16, heads of 128), at the 1.55 GHz that the power cap leaves.
template <bool BF16, int D>
__global__ void __launch_bounds__(kThreads, 1) attention_tiles_kernel(const AttentionParams p) {
  using Sh = Shared<D>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ unsigned long long s_scan[kThreads / 32], s_begin, s_tiles[kThreads / 32];
  __shared__ uint32_t s_tmem, s_failed, s_status;
  __shared__ int s_found;
  launch_dependents();
  wait_for_prior_grids();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  if (tid == kThreads - 1) s_status = *static_cast<volatile unsigned int*>(p.status);  // in the last warp, which has the fewest requests
  const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
  unsigned char* const smem_at = smem_raw + (smem - smem_addr(smem_raw));

  // ---- this CTA's share ----
  unsigned long long* const s_units = reinterpret_cast<unsigned long long*>(smem_at);
  for (int i = warp; i < p.requests; i += kThreads / 32) {
    const Request r = request_of(p, i);
    const uint32_t rows = static_cast<uint32_t>(r.rows) * static_cast<uint32_t>(p.group);
    unsigned long long sum = 0;
    for (uint32_t row0 = static_cast<uint32_t>(lane) * kTilesRows; row0 < rows; row0 += 32u * kTilesRows) sum += steps_of(r, rows, row0, p) + kTileSteps;
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(kFull, sum, d);
    if (lane == 0) s_units[i] = sum;                       // of one key head
  }
  if (tid == 0) {
    s_failed = 0u;
    s_found = 0;
    s_begin = 0;
    const uint32_t bars = smem + Sh::kBars;
#pragma unroll
    for (int i = 0; i < kBarCount; ++i) bar_init(bars + 8 * i, arrivals_of(i));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  __syncthreads();
  unsigned long long total;
  unsigned int ctas;
  Place place;
  {
    const int per = (p.requests + kThreads - 1) / kThreads;
    const int i0 = min(tid * per, p.requests), i1 = min(i0 + per, p.requests);
    unsigned long long mine = 0, tiles = 0;
    for (int i = i0; i < i1; ++i) {
      mine += s_units[i] * static_cast<unsigned>(p.kv_heads);
      tiles += static_cast<unsigned long long>(request_of(p, i).tiles(kTilesRows, p)) * static_cast<unsigned>(p.kv_heads);
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) tiles += __shfl_xor_sync(kFull, tiles, d);
    unsigned long long in = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const unsigned long long up = __shfl_up_sync(kFull, in, d);
      if (lane >= d) in += up;
    }
    if (lane == 31) {
      s_scan[warp] = in;
      s_tiles[warp] = tiles;
    }
    __syncthreads();
    unsigned long long at = in - mine;
    total = 0;
    tiles = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) at += s_scan[w];
      total += s_scan[w];
      tiles += s_tiles[w];
    }
    ctas = static_cast<unsigned int>(min(static_cast<unsigned long long>(gridDim.x), min(total, kMostParts * tiles)));
    if (blockIdx.x >= ctas || s_status != TSQ_OK) return;
    place.unit = scaled(blockIdx.x, total, ctas);
    place.end = scaled(blockIdx.x + 1, total, ctas);
    for (int i = i0; i < i1; ++i) {
      const unsigned long long n = s_units[i] * static_cast<unsigned>(p.kv_heads);
      if (at <= place.unit && place.unit < at + n) {
        s_found = i;
        s_begin = at;
      }
      at += n;
    }
    __syncthreads();
  }
  {
    place.request = s_found;
    place.r = request_of(p, place.request);
    place.rows = static_cast<uint32_t>(place.r.rows) * static_cast<uint32_t>(p.group);
    const unsigned long long of_head = s_units[place.request], in = place.unit - s_begin;
    place.head = static_cast<int>(in / of_head);
    unsigned long long rest = in % of_head;                // steps of this head's tiles in front of `unit`
    // every warp by itself: 32 tiles at a time
    int tile = 0;
    for (;;) {
      const uint32_t row0 = static_cast<uint32_t>(tile + lane) * kTilesRows;
      const int n = row0 < place.rows ? steps_of(place.r, place.rows, row0, p) + kTileSteps : 0;
      int upto = n;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int up = __shfl_up_sync(kFull, upto, d);
        if (lane >= d) upto += up;
      }
      const uint32_t past = __ballot_sync(kFull, static_cast<unsigned long long>(upto) > rest);
      if (past != 0u) {
        const int l = __ffs(static_cast<int>(past)) - 1;
        rest -= __shfl_sync(kFull, upto - n, l);
        tile += l;
        break;
      }
      rest -= __shfl_sync(kFull, upto, 31);
      tile += 32;
      if (static_cast<uint32_t>(tile) * kTilesRows >= place.rows) {  // not reached: the request has the unit
        tile = 0;
        rest = 0;
        break;
      }
    }
    place.tile = tile;
    place.from = static_cast<int>(rest);
    place.before = 0;
    place.take(p);
    if (place.k1 == place.k0 && !place.next(p)) return;
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tm_fence_before();
  __syncthreads();
  tm_fence_after();
  const uint32_t tmem = s_tmem, bars = smem + Sh::kBars;
  bool ok = true;
  // a wait that runs out ends the warp's work, and the others' waits run out in turn
  auto wait = [&](int bar, uint32_t parity) {
    ok = __all_sync(kFull, ok && bar_wait(bars + 8 * bar, parity));
    return ok;
  };

  if (warp < 8) {
    // ---- softmax ----
    regs_up<kSoftmaxRegs>();
    const int t = warp / 4, row = tid % 128;
    const uint32_t lanes = static_cast<uint32_t>(warp % 4) << 21;  // lane 32 * (warp % 4) in the upper half of an address
    const uint32_t s_at = tmem + lanes + 128 * t, o_at = tmem + lanes + 256 + D * t;
    uint32_t count = 0;                                    // steps of this group so far
    const uint32_t group = static_cast<uint32_t>(p.group);
    // whether rows lie on 32-byte boundaries
    const bool q_sectors = ((reinterpret_cast<uintptr_t>(p.q) | static_cast<uintptr_t>(2 * p.q_stride)) & 31u) == 0;
    const bool out_sectors = ((reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(2 * p.out_stride)) & 31u) == 0;
    // the thread's row of a tile, brought to binary16 by a power of two; the inverse is returned
    auto load_query = [&](const Place& at) {
      const uint32_t row0 = static_cast<uint32_t>(at.tile) * kTilesRows + 128u * t;
      float factor = 1.0f;
      if (row0 >= at.rows || at.limit(t, p) <= at.k0) return factor;
      const bool live = row0 + row < at.rows;
      const uint32_t in = live ? row0 + row : row0, token = in / group, query_head = at.head * group + (in - token * group);
      const uint16_t* const from = static_cast<const uint16_t*>(p.q) + (at.r.start + token) * p.q_stride + static_cast<long long>(query_head) * D;
      uint32_t top = 0u;
      uint4 v[D / 8];
      if (q_sectors) {                                     // whole sectors
#pragma unroll
        for (int k = 0; k < D / 8; k += 2) load_sector(v[k], v[k + 1], from + 8 * k);
      } else {
#pragma unroll
        for (int k = 0; k < D / 8; ++k) v[k] = reinterpret_cast<const uint4*>(from)[k];
      }
      if (!live) {
#pragma unroll
        for (int k = 0; k < D / 8; ++k) v[k] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < D / 8; ++k)
        top = __vmaxu2(__vmaxu2(top, v[k].x & 0x7fff7fffu), __vmaxu2(v[k].y & 0x7fff7fffu, __vmaxu2(v[k].z & 0x7fff7fffu, v[k].w & 0x7fff7fffu)));
      const float power = row_power(Elem<BF16>::pattern_f32(max(top & 0xffffu, top >> 16)), factor);
      const float sign = p.scale_log2 < 0.0f ? -power : power;  // the scores' factors are not negative
      unsigned char* const q_at = smem_at + Sh::kQ + t * Sh::kOperand + row * 128;
#pragma unroll
      for (int k = 0; k < D / 8; ++k) {
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        uint32_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = pack_half2(Elem<BF16>::lo_f32(w[e]) * sign, Elem<BF16>::hi_f32(w[e]) * sign);
        *reinterpret_cast<uint4*>(q_at + (k / 8) * kHalf + (((k % 8) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
      }
      fence_proxy_async_smem();
      bar_arrive(bars + 8 * (kQFull + t));
      return factor;
    };
    float factor = load_query(place);
    Place next = place;
    bool more = true;
    for (; more && ok; place = next) {
      const int limit = place.limit(t, p);
      const uint32_t row0 = static_cast<uint32_t>(place.tile) * kTilesRows + 128u * t;
      const bool mine = row0 < place.rows, any = mine && limit > place.k0;  // the group has rows of the tile; the CTA has steps that they see
      const int rows = mine ? static_cast<int>(min(128u, place.rows - row0)) : 1;
      const bool live = row < rows;
      const uint32_t at = row0 + min(row, rows - 1), token = at / group, query_head = place.head * group + (at - token * group);
      float m = 0.0f, l = 0.0f;
      bool have = false, settled = false;                  // the row has a reference; every row of the warp has one below kNearReference
      if (any) {
        const float by_scale = factor * fabsf(p.scale_log2);
        const int seen = place.r.seen(static_cast<int>(token)), seen_first = place.r.seen(static_cast<int>(row0 / group));
        uint32_t scales = static_cast<uint32_t>(place.before) % kMeta;
        for (int j = place.k0; j < limit; ++j, ++count, scales = (scales + 1) % kMeta) {
          const bool mask = (j + 1) * kKeys > seen_first;  // as far as the group's first row sees
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            if (!wait(kSFull + 2 * t + h, count & 1u)) break;
            tm_fence_after();
            const uint32_t at_half = s_at + 64 * h, factors = smem + Sh::kScales + (scales * kGranules + 4 * h) * 16;
            const int left = seen - j * kKeys - 64 * h;    // keys of the half that the row sees
            uint32_t a[32], b[32], w[32];
            tm_load32(a, at_half);
            tm_load32(b, at_half + 32);
            tm_wait_ld(a);
            tm_wait_ld(b);
            float sum = 0.0f, most_weight = 0.0f;
            // once a row has its reference its weights are formed at once, and again only if sixteen neighbours' sum came out above 2^12: no weight is above that in
            // binary16, which goes to 65504
            bool again = !settled;
            if (settled) {
              sum = mask ? weights_of<true, false>(a, b, w, factors, by_scale, m, most_weight, left) : weights_of<false, false>(a, b, w, factors, by_scale, m, most_weight, 64);
              again = __any_sync(kFull, most_weight > 4096.0f);
            }
            if (again) {
              const float most = mask ? fmaxf(top_score<true>(a, factors, by_scale, left), top_score<true>(b, factors + 32, by_scale, left - 32))
                                      : fmaxf(top_score<false>(a, factors, by_scale, 64), top_score<false>(b, factors + 32, by_scale, 64));
              float by = 1.0f;
              if (have ? most > m + 8.0f : most > -INFINITY) {
                by = have ? exp2_fast(m - most) : 0.0f;
                m = most;
                have = true;
              }
              settled = __all_sync(kFull, have && fabsf(m) < kNearReference);
              l *= by;
              if (j > place.k0 || h > 0) {                 // the sums so far follow the reference
                if (!wait(kODone + 2 * t + (h ^ 1), (h > 0 ? count : count - 1u) & 1u)) break;
                tm_fence_after();
#pragma unroll 1
                for (int d = 0; d < D; d += 16) {
                  uint32_t o[16];
                  tm_load16(o, o_at + d);
                  tm_wait_ld(o);
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                  tm_store16(o_at + d, o);
                }
              }
              sum = weights_of<true, true>(a, b, w, factors, by_scale, m, most_weight, mask ? left : 64);
            }
            l += sum;
            tm_store32(at_half, w);                        // in the place of scores, which have all been read
            tm_wait_st();
            tm_fence_before();
            bar_arrive(bars + 8 * (kPReady + 2 * t + h));
          }
          if (!ok) break;
        }
      }
      // the next tile's queries, while the last products are on their way: those with the scores have all ended
      more = next.next(p);
      if (more && ok) factor = load_query(next);
      if (!mine || !ok) continue;
      if (any) {
        if (!wait(kODone + 2 * t + 1, (count - 1u) & 1u)) break;
        tm_fence_after();
      }
      // ---- the row, or its part ----
      uint16_t* const to = static_cast<uint16_t*>(p.out) + (place.r.start + token) * p.out_stride + static_cast<long long>(query_head) * D;
      if (place.k0 == 0 && place.k1 == place.steps) {
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 1
        for (int d = 0; d < D; d += 32) {
          uint32_t o[32];
          tm_load32(o, o_at + d);
          tm_wait_ld(o);
          if (live) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
              uint32_t w[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) w[k] = Elem<BF16>::pack_rn(__uint_as_float(o[e + 2 * k]) * by, __uint_as_float(o[e + 2 * k + 1]) * by);
              store_sector(to + d + e, w, out_sectors);
            }
          }
        }
        tm_fence_before();
        continue;
      }
      // a slot holds columns of 128 rows: maxima, sums, then the dimensions
      constexpr long long kSlot = 128ll * (D + 2);
      float* const slot = p.partials + (4ll * blockIdx.x + 2 * t + (place.k0 > 0 ? 0 : 1)) * kSlot + row;
      slot[0] = l != 0.0f ? m : -INFINITY;                  // a row whose scores are no numbers has a sum that is none
      slot[128] = l;
      if (any) {
#pragma unroll 1
        for (int d = 0; d < D; d += 32) {
          uint32_t o[32];
          tm_load32(o, o_at + d);
          tm_wait_ld(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) slot[128 * (2 + d + e)] = __uint_as_float(o[e]);
        }
        tm_fence_before();
      }
      const unsigned long long tile_begin = place.unit - place.from + kTileSteps;  // its first step
      const int first = owner_of(tile_begin, total, ctas), last = owner_of(tile_begin + place.steps - 1, total, ctas);
      __threadfence();
      __syncwarp();
      unsigned int done = 0u;                              // a warp's rows by themselves
      if (lane == 0) done = atomicInc(p.counters + 8 * first + warp, static_cast<unsigned>(last - first));
      if (__shfl_sync(kFull, done, 0) == static_cast<unsigned>(last - first)) {
        __threadfence();
        // two parts and 32 dimensions at a time, without a branch between the loads, so that all of them are on their way; behind the last part its data again, not counted
        const auto part_at = [&](int n) { return p.partials + (4ll * min(n, last) + 2 * t + (min(n, last) == first ? 1 : 0)) * kSlot + row; };
        float top = -INFINITY, all = 0.0f;
#pragma unroll 4
        for (int n = first; n <= last; ++n) top = fmaxf(top, __ldcg(part_at(n)));
#pragma unroll 1
        for (int d = 0; d < D; d += 32) {
          float o[32];
          all = 0.0f;
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.0f;
#pragma unroll 1
          for (int n = first; n <= last; n += 2) {
            const float *const p0 = part_at(n), *const p1 = part_at(n + 1);
            const float m0 = __ldcg(p0), m1 = n < last ? __ldcg(p1) : -INFINITY, l0 = __ldcg(p0 + 128), l1 = __ldcg(p1 + 128);
            float x0[32], x1[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              x0[e] = __ldcg(p0 + 128 * (2 + d + e));
              x1[e] = __ldcg(p1 + 128 * (2 + d + e));
            }
            // a part of maximum -Inf has seen nothing: what stands in its slot does not count, whatever it is
            const float w0 = m0 == -INFINITY ? 0.0f : exp2_fast(m0 - top), w1 = m1 == -INFINITY ? 0.0f : exp2_fast(m1 - top);
            all += (m0 == -INFINITY ? 0.0f : l0 * w0) + (m1 == -INFINITY ? 0.0f : l1 * w1);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] += (m0 == -INFINITY ? 0.0f : x0[e] * w0) + (m1 == -INFINITY ? 0.0f : x1[e] * w1);
          }
          const float by = all == 0.0f ? 0.0f : 1.0f / all;
          if (live) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
              uint32_t w[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) w[k] = Elem<BF16>::pack_rn(o[e + 2 * k] * by, o[e + 2 * k + 1] * by);
              store_sector(to + d + e, w, out_sectors);
            }
          }
        }
      }
    }
    regs_back<kSoftmaxRegs>(warp / 4, !ok, &s_failed);
  } else if (warp < 16) {
    // ---- codes to binary16: a warpgroup for the keys, one for the values ----
    regs_down<kWidenRegs>();
    constexpr int kChunks = D / 16;                        // 16-byte chunks of a token's codes
    constexpr int kItems = kKeys * kChunks / 128;          // per thread and step
    const bool values = warp >= 12;
    const int w = warp % 4, in_group = tid % 128;
    const int8_t* const codes = values ? p.v_codes : p.k_codes;
    const int full = values ? kVFull : kKFull, free = values ? kVFree : kKFree;
    // eight neighbouring lanes write four chunks of two neighbouring tokens: the swizzle puts those in different banks
    const int token0 = D == 128 ? w * 4 + (lane >> 4) * 2 + ((lane >> 2) & 1) : w * 8 + (lane >> 2);
    const int chunk = D == 128 ? (lane & 3) | ((lane >> 3) & 1) << 2 : lane & 3;
    unsigned char* const to = smem_at + (values ? Sh::kV : Sh::kK) + (chunk / 4) * kHalf;
    const bool has_scale = !values && in_group < kGranules;  // the keys' group leaves the scales too, a thread for each granule
    uint32_t n = 0;                                        // steps so far
    uint4 raw[kItems];
    float4 scale = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // pages of the next step's granules, -1 where there is none: every thread reads those of its own tokens (one lane for each granule and shuffles: 16 requests of 8000 tokens,
    // 64 rows 150 -> 217 us, 5 requests in chunks 366 -> 420, although fewer instructions)
    int pages[kItems], scale_page = -1;
    auto page_at = [&](int j, int granule) {
      const int token = j * kKeys + 16 * granule;
      if (token >= place.r.keys) return -1;
      return p.table[static_cast<long long>(place.request) * p.table_pages + (token >> p.page_shift)];
    };
    auto fetch_pages = [&](int j) {
#pragma unroll
      for (int it = 0; it < kItems; ++it) pages[it] = page_at(j, (token0 + it * (128 / kChunks)) / 16);
      if (has_scale) scale_page = page_at(j, in_group);
    };
    auto fetch = [&](int j) {
#pragma unroll
      for (int it = 0; it < kItems; ++it) {
        const int token = j * kKeys + token0 + it * (128 / kChunks);
        raw[it] = make_uint4(0u, 0u, 0u, 0u);
        if (static_cast<unsigned>(pages[it]) < static_cast<unsigned>(p.pages))
          raw[it] = *(reinterpret_cast<const uint4*>(codes + (((static_cast<long long>(pages[it]) * p.kv_heads + place.head) << p.page_shift) +
                                                              (token & ((1 << p.page_shift) - 1))) * D) + chunk);
      }
      if (has_scale) {
        scale = make_float4(0.0f, -INFINITY, 0.0f, 0.0f);  // nothing of a page that is not there is seen
        if (static_cast<unsigned>(scale_page) < static_cast<unsigned>(p.pages)) {
          const long long page_head = static_cast<long long>(scale_page) * p.kv_heads + place.head;
          const float vs = p.v_scale[page_head];
          scale = make_float4(p.k_scale[page_head], log2_of_scale(vs), inverse_of_scale(vs), 0.0f);
        }
      }
    };
    int j = place.k0;
    bool more = true;
    fetch_pages(j);
    fetch(j);
    while (more) {
      if (++j >= place.k1) {                               // the step behind this one
        more = place.next(p);
        j = place.k0;
      }
      if (more) fetch_pages(j);
      const uint32_t buffer = n & 1u;
      if (!wait(free + buffer, ((n >> 1) & 1u) ^ 1u)) break;
      if (has_scale) reinterpret_cast<float4*>(smem_at + Sh::kScales)[(n % kMeta) * kGranules + in_group] = scale;
#pragma unroll
      for (int it = 0; it < kItems; ++it) {
        const int token = token0 + it * (128 / kChunks);
        const uint32_t u[4] = {raw[it].x ^ 0x80808080u, raw[it].y ^ 0x80808080u, raw[it].z ^ 0x80808080u, raw[it].w ^ 0x80808080u};
        unsigned char* const at = to + buffer * Sh::kOperand + token * 128;
        const int c = 2 * (chunk % 4), x = token & 7;
        *reinterpret_cast<uint4*>(at + ((c ^ x) << 4)) = make_uint4(widen_lo(u[0]), widen_hi(u[0]), widen_lo(u[1]), widen_hi(u[1]));
        *reinterpret_cast<uint4*>(at + (((c + 1) ^ x) << 4)) = make_uint4(widen_lo(u[2]), widen_hi(u[2]), widen_lo(u[3]), widen_hi(u[3]));
      }
      fence_proxy_async_smem();
      bar_arrive(bars + 8 * (full + buffer));
      if (more) fetch(j);
      ++n;
    }
    regs_back<kWidenRegs>(warp / 4, !ok, &s_failed);
  } else {
    regs_down<kProductRegs>();
    if (warp < 18) {
      // ---- products: a warp for each group ----
      const int t = static_cast<int>(uniform(warp - 16));
      const uint32_t leader = elected(), base = uniform(smem), bar = uniform(bars), tm = uniform(tmem);
      constexpr uint32_t kScores = product_of(kKeys / 2, false), kSums = product_of(D, true);
      uint32_t n = 0, count = 0, tiles = 0;                  // steps; steps and tiles of the group
      bool issued = false;
      // scores of 64 of the keys in buffer `buffer`
      auto scores = [&](uint32_t buffer, int h) {
        tm_fence_after();
        issued = true;
        const uint64_t queries = operand(base + Sh::kQ + t * Sh::kOperand, 16, 1024), keys = operand(base + Sh::kK + buffer * Sh::kOperand + h * (kHalf / 2), 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          constexpr uint32_t kUnit = 16;                     // bytes that a descriptor's address counts
          const uint32_t off = ((k / 4) * kHalf + (k % 4) * 32) / kUnit;
          product_ss(leader, tm + 128 * t + 64 * h, queries + off, keys + off, kScores, k > 0);
        }
        tm_commit(leader, bar + 8 * (kSFull + 2 * t + h));
        if (h == 1) tm_commit(leader, bar + 8 * (kKFree + buffer));
      };
      do {
        const int limit = place.limit(t, p);
        int j = place.k0;
        if (j < limit) {
          if (!wait(kQFull + t, tiles & 1u) || !wait(kKFull + (n & 1u), (n >> 1) & 1u)) break;
          ++tiles;
          for (int h = 0; h < 2; ++h) {
            // the weights in the scores' place have been used
            if (count > 0 && !wait(kODone + 2 * t + h, (count - 1u) & 1u)) break;
            scores(uniform(n & 1u), h);
          }
        }
        for (; j < limit && ok; ++j) {
          const uint32_t buffer = uniform(n & 1u);
          if (!wait(kVFull + buffer, (n >> 1) & 1u)) break;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!wait(kPReady + 2 * t + h, count & 1u)) break;
            tm_fence_after();
            const uint64_t values = operand(base + Sh::kV + buffer * Sh::kOperand + h * (kHalf / 2), kHalf, 1024);
            const uint32_t add = uniform(j > place.k0 || h > 0);
#pragma unroll
            for (int k = 0; k < kKeys / 32; ++k)             // 16 tokens: 2048 bytes
              product_ts(leader, tm + 256 + D * t, tm + 128 * t + 64 * h + 8 * k, values + 128 * k, kSums, add != 0u || k > 0);
            tm_commit(leader, bar + 8 * (kODone + 2 * t + h));
            if (h == 1) tm_commit(leader, bar + 8 * (kVFree + buffer));
            if (j + 1 < limit) {
              if (h == 0 && !wait(kKFull + (buffer ^ 1u), ((n + 1u) >> 1) & 1u)) break;
              if (!wait(kODone + 2 * t + h, count & 1u)) break;
              scores(buffer ^ 1u, h);
            }
          }
          ++n;
          ++count;
        }
        // steps that only the other group has: the buffers are not waited for on this one's account
        for (; j < place.k1 && ok; ++j, ++n) {
          const uint32_t buffer = n & 1u, phase = (n >> 1) & 1u;
          if (!wait(kKFull + buffer, phase)) break;
          bar_arrive(bars + 8 * (kKFree + buffer));
          if (!wait(kVFull + buffer, phase)) break;
          bar_arrive(bars + 8 * (kVFree + buffer));
          __syncwarp();
        }
      } while (ok && place.next(p));
      // everything issued has ended before the tensor memory is given back, wherever the loops were left: a commit stands for all of the thread's products before it
      if (issued) {
        tm_commit(leader, bar + 8 * (kEnd + t));
        if (!bar_wait(bars + 8 * (kEnd + t), 0u)) ok = false;
      }
      ok = __all_sync(kFull, ok);
    }
    regs_back<kProductRegs>(4, !ok, &s_failed);
  }
  tm_fence_before();
  __syncthreads();
  tm_fence_after();
  if (threadIdx.x / 32 == 16) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(*static_cast<volatile uint32_t*>(&s_tmem)) : "memory");
  if (threadIdx.x == 0 && s_failed != 0u) atomicExch(p.status, static_cast<unsigned>(TSQ_ERR_TIMEOUT));
}

template <bool BF16, int D>
cudaError_t launch(const AttentionParams& p, int ctas, cudaStream_t stream) {
  constexpr int bytes = Shared<D>::kBytes + 1024;
  static_assert(Shared<D>::kScales >= 8 * kMaxRequests, "the unit counts fit in front of the scales");
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_shared(attention_tiles_kernel<BF16, D>, bytes, done);
  if (e != cudaSuccess) return e;
  return launch_overlapped(attention_tiles_kernel<BF16, D>, ctas, kThreads, bytes, stream, p);
}

}  // namespace

cudaError_t launch_attention_tiles(const AttentionParams& p, bool bf16, int head_dim, int sms, cudaStream_t stream) {
  if (head_dim == 128) return bf16 ? launch<true, 128>(p, sms, stream) : launch<false, 128>(p, sms, stream);
  return bf16 ? launch<true, 64>(p, sms, stream) : launch<false, 64>(p, sms, stream);
}

}  // namespace tsq
