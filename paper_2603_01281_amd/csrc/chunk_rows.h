// Attention of new tokens over a cache of pages, few rows at a time: pieces that the bf16 and the fp32 kernel share.
#pragma once
#include <type_traits>

#include "paged.h"

namespace seka {

constexpr float kRowSlack = 8.f;         // a row's reference exponent trails its maximum by at most this (base 2)
constexpr float kRowLow = -1e30f;        // reference of a row that has seen nothing

// Merged state of four output columns of a row: the output itself if the item has its rows to itself, else a partial state.
template <typename T, int D>
__device__ __forceinline__ void row_emit(const ChunkArgs& a, const ChunkItem& it, int h, int row, int d, float m, float l, f32x4 o) {
  if (it.splits > 1) {
    float* dst = a.part + (((size_t)blockIdx.x * a.Hkv + h) * a.p.R + (row - it.rc * a.p.R)) * (D + 4);
    *reinterpret_cast<f32x4*>(dst + d) = o;
    if (d == 0) {
      dst[D] = m;
      dst[D + 1] = l;
    }
    return;
  }
  const int G = a.p.G, i = row / G, hq = h * G + row - i * G;
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  T* O = static_cast<T*>(a.O) + ((size_t)(it.e.row0 + i) * a.Hq + hq) * D + d;
  if constexpr (sizeof(T) == 2) {
    bf16x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (__bf16)(o[k] * inv);
    *reinterpret_cast<bf16x4*>(O) = v;
  } else {
    *reinterpret_cast<f32x4*>(O) = o * inv;
  }
  if (a.lse && d == 0) a.lse[(size_t)hq * a.r.total + it.e.row0 + i] = some ? m * 0.6931471805599453f + logf(l) : -INFINITY;
}

// The waves' states of 16 rows (sm_o [wave][16][D + 4], sm_ml [wave][16][2]) to row_emit; row0: the first of them, rows of the request.
template <typename T, int D, int NW>
__device__ __forceinline__ void merge_waves(const ChunkArgs& a, const ChunkItem& it, int h, int row0, const float* sm_o, const float (*sm_ml)[16][2]) {
  const int rows = min(16, min((it.rc + 1) * a.p.R, it.e.n * a.p.G) - row0);
  for (int idx = threadIdx.x; idx < rows * (D / 4); idx += 64 * NW) {
    const int r = idx / (D / 4), d = idx % (D / 4) * 4;
    float mm = sm_ml[0][r][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) mm = fmaxf(mm, sm_ml[w][r][0]);
    float ll = 0.f;
    f32x4 oo = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_ml[w][r][0] - mm);
      ll += sm_ml[w][r][1] * f;
      oo += *reinterpret_cast<const f32x4*>(sm_o + (w * 16 + r) * (D + 4) + d) * f;
    }
    row_emit<T, D>(a, it, h, row0 + r, d, mm, ll, oo);
  }
}

// Queries have arrived here: their registers are not waited for in the loop, which would wait for the loads of the next keys with them.
template <typename V, int A, int B>
__device__ __forceinline__ void row_arrived(V (&q)[A][B]) {
#pragma unroll
  for (int a = 0; a < A; ++a)
#pragma unroll
    for (int b = 0; b < B; ++b) asm volatile("" : "+v"(q[a][b]));
}

// What the joining kernel has to know of an item: how many ranges its chunk has (0: not the chunk's first, or no item), where its rows are.
__device__ __forceinline__ void row_describe(const ChunkArgs& a, bool exists, const ChunkItem& it) {
  if (blockIdx.y == 0 && threadIdx.x == 0)
    a.items_of[blockIdx.x] = exists && it.split == 0 ? make_int4(it.splits, it.e.row0, it.e.n, it.rc * a.p.R) : make_int4(0, 0, 0, 0);
}

// The ranges' states of a row: blockIdx = (first item of a chunk, KV head, first row; the next one gridDim.z further).  Groups of D / 4 threads take every
// NJ-th range, four columns to a thread, all of whose loads are issued before the first is used; the groups join in LDS.
constexpr int kMergeThreads = 256, kMaxRanges = 64;
template <typename T, int D>
__global__ __launch_bounds__(kMergeThreads) void chunk_merge_kernel(ChunkArgs a) {
  constexpr int LANES = D / 4, NJ = kMergeThreads / LANES, NI = kMaxRanges / NJ;
  __shared__ f32x4 sm_o[NJ][LANES];
  __shared__ float sm_m[NJ], sm_l[NJ];
  const int4 it = a.items_of[blockIdx.x];
  const int splits = min(it.x, (int)(gridDim.x - blockIdx.x)), h = blockIdx.y, G = a.p.G;
  if (splits <= 1) return;
  const int rows = min(a.p.R, it.z * G - it.w);
  for (int r = blockIdx.z; r < rows; r += gridDim.z) {            // workgroup-uniform
    const int row = it.w + r;
    const int c = threadIdx.x % LANES, j = threadIdx.x / LANES;
    const size_t stride = (size_t)a.Hkv * a.p.R * (D + 4);
    const float* src = a.part + ((size_t)blockIdx.x * a.Hkv + h) * a.p.R * (D + 4) + (size_t)r * (D + 4);
    float mv[NI], lv[NI];
    f32x4 ov[NI];
    auto gather = [&](auto count) __attribute__((always_inline)) {
      constexpr int N = decltype(count)::value;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float* ps = src + (size_t)min(j + NJ * i, splits - 1) * stride;
        mv[i] = ps[D];
        lv[i] = ps[D + 1];
        ov[i] = *reinterpret_cast<const f32x4*>(ps + 4 * c);
      }
      float m = kRowLow, l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (j + NJ * i < splits) m = fmaxf(m, mv[i]);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (j + NJ * i < splits) {
          const float f = __builtin_amdgcn_exp2f(mv[i] - m);
          l += lv[i] * f;
          o += ov[i] * f;
        }
      sm_o[j][c] = o;
      if (c == 0) {
        sm_m[j] = m;
        sm_l[j] = l;
      }
    };
    if (splits <= NJ) gather(std::integral_constant<int, 1>{});
    else if (splits <= 2 * NJ) gather(std::integral_constant<int, 2>{});
    else gather(std::integral_constant<int, NI>{});
    __syncthreads();
    if (j == 0) {
      float m = sm_m[0], l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 1; k < NJ; ++k) m = fmaxf(m, sm_m[k]);
#pragma unroll
      for (int k = 0; k < NJ; ++k) {
        const float f = __builtin_amdgcn_exp2f(sm_m[k] - m);
        l += sm_l[k] * f;
        o += sm_o[k][c] * f;
      }
      const int i = row / G, hq = h * G + row % G;
      const bool some = l > 0.f || l != l;
      const float inv = some ? 1.f / l : 0.f;
      T* O = static_cast<T*>(a.O) + ((size_t)(it.y + i) * a.Hq + hq) * D + 4 * c;
      if constexpr (sizeof(T) == 2) {
        bf16x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (__bf16)(o[k] * inv);
        *reinterpret_cast<bf16x4*>(O) = v;
      } else {
        *reinterpret_cast<f32x4*>(O) = o * inv;
      }
      if (a.lse && c == 0) a.lse[(size_t)hq * a.r.total + it.y + i] = some ? m * 0.6931471805599453f + logf(l) : -INFINITY;
    }
    __syncthreads();                         // the next row's states
  }
}

// rows: of a chunk that exist, at most
template <typename T, int D>
void launch_chunk_merge(const ChunkArgs& a, int items, int rows, hipStream_t s) {
  if (a.p.max_splits <= 1) return;
  const int z = (long long)items * a.Hkv * rows <= 16384 || rows < 16 ? rows : 16;       // workgroups beyond that have several rows each
  hipLaunchKernelGGL((chunk_merge_kernel<T, D>), dim3(items, a.Hkv, z), dim3(kMergeThreads), 0, s, a);
}

// How a call with few rows is launched: waves per workgroup, tiles of 16 rows, rows that a chunk can have, items.
struct RowPlan {
  ChunkPlan p;
  int waves, rows16, rows, items;
};
hipError_t launch_chunk_bf16(const ChunkArgs& a, int D, const RowPlan& r, hipStream_t s);
hipError_t launch_chunk_f32(const ChunkArgs& a, int D, const RowPlan& r, hipStream_t s);

}  // namespace seka
