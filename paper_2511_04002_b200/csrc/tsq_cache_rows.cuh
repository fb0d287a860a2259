// What the kernels of attention over the paged cache for few query rows share, whatever width its codes have: products, a CTA's share of the work, the queries, and a tile's end.
#ifndef TSQ_CACHE_ROWS_CUH_
#define TSQ_CACHE_ROWS_CUH_

#include "tsq_cache.h"
#include "tsq_cache_device.cuh"
#include "tsq_device.cuh"

namespace tsq {

constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = 32 * kRowsWarps;
constexpr int kRowsFanIn = 16;               // parts of a tile that are added up at once

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

// Where a tile of 8 NT rows has the four warps' sums in shared memory, once its stages have been read.
template <int D, int NT>
struct RowsSums {
  static constexpr int kRows = 8 * NT;
  static constexpr int kRowFloats = D + 36;              // a row of a warp's sums: four floats more behind each eighth, and four at the end
  static constexpr int kSums = kRowsWarps * kRows * kRowFloats * 4;
  static constexpr int kBytes = kSums + kRowsWarps * kRows * 8;
};

// The CTA's share of the units [unit, end) of `total`, and the request that has its first unit; `rest` units of it lie in front.
struct Share {
  unsigned long long total, unit, end, rest;
  unsigned int ctas;
  int request;
};
// False: the CTA has none, or the workspace is not to be used.  Every thread sums its requests' units, and the one whose sums reach past the first unit tells the others.
template <int ROWS, int UNIT, int MORE>
__device__ __forceinline__ bool share_of(const AttentionParams& p, Share& s) {
  __shared__ unsigned long long s_scan[kRowsWarps], s_begin;
  __shared__ int s_found;
  __shared__ unsigned int s_status;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const unsigned int status = *static_cast<volatile unsigned int*>(p.status);  // one thread's is used, behind a barrier: on its way with the requests
  const int per = (p.requests + kRowsThreads - 1) / kRowsThreads;
  const int i0 = min(tid * per, p.requests), i1 = min(i0 + per, p.requests);
  unsigned long long mine = 0, n = 0;
  for (int i = i0; i < i1; ++i) {
    n = request_of(p, i).units(ROWS, UNIT, MORE, p);
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
  s.total = 0;
#pragma unroll
  for (int w = 0; w < kRowsWarps; ++w) {
    if (w < warp) at += s_scan[w];
    s.total += s_scan[w];
  }
  s.ctas = s.total < gridDim.x ? static_cast<unsigned int>(s.total) : gridDim.x;
  if (blockIdx.x >= s.ctas || s_status != TSQ_OK) return false;
  s.unit = scaled(blockIdx.x, s.total, s.ctas);
  s.end = scaled(blockIdx.x + 1, s.total, s.ctas);
  if (at <= s.unit && s.unit < at + mine) {
    for (int i = i0; i < i1; ++i) {
      if (per > 1) n = request_of(p, i).units(ROWS, UNIT, MORE, p);
      if (s.unit < at + n) {
        s_found = i;
        s_begin = at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  s.request = s_found;
  s.rest = s.unit - s_begin;
  return true;
}

// A tile's end: the four warps' references m, sums l and accumulators (those of thread (g, c): rows 8 t + 2 c and + 1, dimensions g * D / 8 + 2 d of tile d in [0] and [1], + 1 in [2] and [3]) are
// brought together, and the rows written; where other CTAs have units of the tile too (`shared`; the units first_unit .. last_unit of the call), by the one that comes last.
template <bool BF16, int D, int NT>
__device__ __forceinline__ void finish_tile(const AttentionParams& p, const Share& s, const Request& r, int head, int row0, int rows, bool shared, unsigned long long first_unit,
                                            unsigned long long last_unit, unsigned char* smem, const float (&m)[NT][2], const float (&l)[NT][2],
                                            const float (&acc)[NT][D / 16][4]) {
  using L = RowsSums<D, NT>;
  constexpr int kTiles = D / 16;
  __shared__ unsigned int s_last;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, c = lane % 4;
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
  constexpr int kParts = kRowsThreads / L::kRows, kDims = D / kParts;  // threads of a row, and what each has of it
  const int row = tid / kParts, d0 = tid % kParts * kDims, padded = d0 + d0 / (D / 8) * 4;
  float o[kDims], top = -INFINITY, all = 0.0f;
#pragma unroll
  for (int w = 0; w < kRowsWarps; ++w) top = fmaxf(top, stats[w * L::kRows + row].x);
#pragma unroll
  for (int d = 0; d < kDims; ++d) o[d] = 0.0f;
#pragma unroll
  for (int w = 0; w < kRowsWarps; ++w) {
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
  if (shared) {                            // other CTAs have units of this tile
    // Parts are added up sixteen at a time by the CTA that comes last of the sixteen, their sums likewise: the order does not depend on who comes when.
    const int first = owner_of(first_unit, s.total, s.ctas), parts = owner_of(last_unit, s.total, s.ctas) - first + 1;
    constexpr int kSlot = L::kRows * (D + 2);
    const auto slot_of = [&](int n) { return p.partials + (2ll * (first + n) + (n == 0 ? 1 : 0)) * kSlot; };
    int part = static_cast<int>(blockIdx.x) - first;
    unsigned int* counters = p.counters;
    for (int stride = 1; stride < parts && write; stride *= kRowsFanIn, counters += gridDim.x) {
      const int begin = part / (kRowsFanIn * stride) * (kRowsFanIn * stride), members = min(kRowsFanIn, (parts - begin + stride - 1) / stride);
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
          float2 st[kRowsFanIn];
#pragma unroll
          for (int n = 0; n < kRowsFanIn; ++n) st[n] = __ldcg(reinterpret_cast<const float2*>(part_at(n) + L::kRows * D) + row);
          top = -INFINITY;
#pragma unroll
          for (int n = 0; n < kRowsFanIn; ++n) {
            if (n >= members) st[n] = make_float2(-INFINITY, 0.0f);
            top = fmaxf(top, st[n].x);
          }
          all = 0.0f;
#pragma unroll
          for (int d = 0; d < kDims; ++d) o[d] = 0.0f;
          constexpr int kBatch = 64 / kDims < kRowsFanIn ? 64 / kDims : kRowsFanIn;
#pragma unroll
          for (int n0 = 0; n0 < kRowsFanIn; n0 += kBatch) {
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

}  // namespace tsq

#endif  // TSQ_CACHE_ROWS_CUH_
