// Attention of new tokens over a cache of pages, few rows at a time: pieces that the bf16 and the fp32 kernel share.
#pragma once
#include "paged.h"

namespace seka {

constexpr int kRowThreads = 64 * kRowWaves;
constexpr float kRowSlack = 8.f;         // a row's reference exponent trails its maximum by at most this (base 2)
constexpr float kRowLow = -1e30f;        // reference of a row that has seen nothing

// Merged state of output column d of a row: the output itself if the item has its rows to itself, else a partial state.
template <typename T, int D>
__device__ __forceinline__ void row_emit(const ChunkArgs& a, const ChunkItem& it, int h, int row, int d, float m, float l, float o) {
  const int G = a.p.G, i = row / G, hq = h * G + row % G;
  if (it.splits == 1) {
    const float v = l > 0.f || l != l ? o / l : 0.f;
    T* O = static_cast<T*>(a.O) + ((size_t)(it.e.row0 + i) * a.Hq + hq) * D + d;
    if constexpr (sizeof(T) == 2) *O = __builtin_bit_cast(T, (__bf16)v);
    else *O = v;
    if (a.lse && d == 0) a.lse[(size_t)hq * a.r.total + it.e.row0 + i] = l > 0.f || l != l ? m * 0.6931471805599453f + logf(l) : -INFINITY;
    return;
  }
  float* dst = a.part + (((size_t)it.index * a.Hkv + h) * a.p.R + (row - it.rc * a.p.R)) * (D + 4);
  dst[d] = o;
  if (d == 0) {
    dst[D] = m;
    dst[D + 1] = l;
  }
}

// The waves' states of 16 rows (sm_o [wave][16][D + 4], sm_ml [wave][16][2]) to row_emit; row0: the first of them, rows of the request.
template <typename T, int D>
__device__ __forceinline__ void merge_waves(const ChunkArgs& a, const ChunkItem& it, int h, int row0, const float* sm_o, const float (*sm_ml)[16][2]) {
  const int rows = min(16, min((it.rc + 1) * a.p.R, it.e.n * a.p.G) - row0);
  for (int idx = threadIdx.x; idx < rows * D; idx += kRowThreads) {
    const int r = idx / D, d = idx % D;
    float mm = sm_ml[0][r][0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) mm = fmaxf(mm, sm_ml[w][r][0]);
    float ll = 0.f, oo = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_ml[w][r][0] - mm);
      ll += sm_ml[w][r][1] * f;
      oo += sm_o[(w * 16 + r) * (D + 4) + d] * f;
    }
    row_emit<T, D>(a, it, h, row0 + r, d, mm, ll, oo);
  }
}

// Partial states of a chunk's ranges, one workgroup per (chunk, KV head); a thread takes four columns of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a) {
  ChunkItem it;
  if (!plan_item<true>(a.r, a.c, a.p, blockIdx.x, it) || it.splits == 1 || it.index + it.splits > a.items) return;
  const int h = blockIdx.y, G = a.p.G;
  const int rows = min(a.p.R, it.e.n * G - it.rc * a.p.R);
  const float* src = a.part + ((size_t)it.index * a.Hkv + h) * a.p.R * (D + 4);
  const size_t stride = (size_t)a.Hkv * a.p.R * (D + 4);
  for (int idx = threadIdx.x; idx < rows * (D / 4); idx += 256) {
    const int r = idx / (D / 4), d = idx % (D / 4) * 4;
    const float* ps = src + (size_t)r * (D + 4);
    float m = kRowLow, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < it.splits; ++s, ps += stride) {
      const float m2 = ps[D], l2 = ps[D + 1];
      const f32x4 o2 = *reinterpret_cast<const f32x4*>(ps + d);
      const float mm = fmaxf(m, m2), f1 = __builtin_amdgcn_exp2f(m - mm), f2 = __builtin_amdgcn_exp2f(m2 - mm);
      m = mm;
      l = l * f1 + l2 * f2;
      o = o * f1 + o2 * f2;
    }
    const int row = it.rc * a.p.R + r, i = row / G, hq = h * G + row % G;
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
}

hipError_t launch_chunk_bf16(const ChunkArgs& a, int D, int rows16, int items, int chunks, hipStream_t s);
hipError_t launch_chunk_f32(const ChunkArgs& a, int D, int rows16, int items, int chunks, hipStream_t s);

}  // namespace seka
