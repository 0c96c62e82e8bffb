// Rotary positions, and their use where new tokens enter a cache of pages.
//
// A pair (x, y) of a head's first 2 half elements at position p turns by p f_i:  (x cos - y sin, y cos + x sin), times a factor.
// f_i p is formed in revolutions in 64 bits and its whole part dropped there: at position 10^6 the angle of the fastest pair in
// 32 bits would be off by 0.03 radians.
//
// HBM-bound: every row is read and written once.  A workgroup takes one token (grid.y: a share of its heads); one sine and cosine
// per pair, which all heads of the token share, go through LDS while the first rows are on their way.  A thread owns whole pairs
// (16 bytes on each side), so input and output may be the same memory.
#include "paged.h"

namespace seka {
namespace {

constexpr int kRotThreads = 256;

template <typename T> struct RotElem;
template <> struct RotElem<uint16_t> {
  static constexpr int V = 8;
  __device__ static float get(uint16_t x) { return bf16_bits_to_float(x); }
  __device__ static uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <> struct RotElem<float> {
  static constexpr int V = 4;
  __device__ static float get(float x) { return x; }
  __device__ static float put(float x) { return x; }
};

template <typename T, bool PAGED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  using E = RotElem<T>;
  constexpr int V = E::V;
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  __shared__ float cs[64], sn[64];
  const int t = blockIdx.x, tid = threadIdx.x;

  // ---- where the token lies ----
  bool owned = true, cached = false;
  int slot = 0, page = 0;
  int pos = 0;
  if (PAGED) {
    // the request is the number of requests that end at or before row t
    int b = 0;
    for (int b0 = 0; b0 < a.r.B; b0 += kRotThreads)
      b += __syncthreads_count(b0 + tid < a.r.B && a.r.cu[min(b0 + tid, a.r.B - 1) + 1] <= t);
    owned = b < a.r.B;
    if (owned) {
      const ChunkExtent e = chunk_extent(a.r, a.c, b);
      const int i = t - e.row0;
      owned = i >= 0 && i < e.n;
      const int j = e.len - e.n + i;
      cached = owned && j >= 0;
      if (cached) {
        page = page_of(a.c, b, j);
        slot = j & ((1 << a.c.shift) - 1);
      }
      pos = j;
    }
    if (!owned) return;                      // the same in every thread
  } else {
    pos = t % a.S;
  }
  if (a.positions) pos = a.positions[t];

  if (tid < a.half) {
    double turn = (double)pos * a.turns[tid];
    turn -= rint(turn);
    float s, c;
    sincospif(2.0f * (float)turn, &s, &c);
    cs[tid] = c * a.factor;
    sn[tid] = s * a.factor;
  }
  __syncthreads();

  // ---- units: V pairs each, then pieces of V elements that are copied ----
  const int dim = 2 * a.half;
  const int nrot = (a.half + V - 1) / V;
  const bool vec_pairs = a.interleaved ? dim % (2 * V) == 0 : a.half % V == 0;
  const int ncopy = (a.D - dim + V - 1) / V;
  const bool vec_copy = dim % V == 0;
  const int per_row = nrot + ncopy;
  const int q_rows = a.Q ? a.Hq : 0, k_rows = a.K ? a.Hkv : 0, v_rows = PAGED ? a.Hkv : 0;
  const int units = (q_rows + k_rows) * per_row;
  const size_t cache_row = ((((size_t)page << a.c.shift) + slot) * a.Hkv) * a.D;
  for (int u = blockIdx.y * kRotThreads + tid; u < units; u += gridDim.y * kRotThreads) {
    const int row = u / per_row, part = u % per_row;
    const bool is_q = row < q_rows;
    const int h = is_q ? row : row - q_rows;
    if (PAGED && !is_q && !cached) continue;
    const T* src = is_q ? static_cast<const T*>(a.Q) + ((size_t)t * a.Hq + h) * a.D : static_cast<const T*>(a.K) + ((size_t)t * a.Hkv + h) * a.D;
    T* dst = is_q ? static_cast<T*>(a.Q_out) + ((size_t)t * a.Hq + h) * a.D
             : PAGED ? static_cast<T*>(a.c.K) + cache_row + (size_t)h * a.D
                     : static_cast<T*>(a.K_out) + ((size_t)t * a.Hkv + h) * a.D;
    if (part >= nrot) {                      // behind the rotated part
      if (src == dst) continue;
      const int e0 = dim + (part - nrot) * V;
      if (vec_copy) {
        *reinterpret_cast<u32x4*>(dst + e0) = *reinterpret_cast<const u32x4*>(src + e0);
      } else {
        for (int e = e0; e < min(e0 + V, a.D); ++e) dst[e] = src[e];
      }
      continue;
    }
    const int p0 = part * V;
    if (vec_pairs) {
      const int i0 = a.interleaved ? 2 * p0 : p0, i1 = a.interleaved ? 2 * p0 + V : a.half + p0;
      u32x4 v0 = *reinterpret_cast<const u32x4*>(src + i0), v1 = *reinterpret_cast<const u32x4*>(src + i1);
      T x[V], y[V];
      __builtin_memcpy(x, &v0, 16);
      __builtin_memcpy(y, &v1, 16);
      if (a.interleaved) {
#pragma unroll
        for (int k = 0; k < V; k += 2) {
          const int p = p0 + k / 2, q = p + V / 2;
          const float x0 = E::get(x[k]), x1 = E::get(x[k + 1]), y0 = E::get(y[k]), y1 = E::get(y[k + 1]);
          x[k] = E::put(x0 * cs[p] - x1 * sn[p]);
          x[k + 1] = E::put(x1 * cs[p] + x0 * sn[p]);
          y[k] = E::put(y0 * cs[q] - y1 * sn[q]);
          y[k + 1] = E::put(y1 * cs[q] + y0 * sn[q]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float x0 = E::get(x[k]), y0 = E::get(y[k]);
          x[k] = E::put(x0 * cs[p0 + k] - y0 * sn[p0 + k]);
          y[k] = E::put(y0 * cs[p0 + k] + x0 * sn[p0 + k]);
        }
      }
      __builtin_memcpy(&v0, x, 16);
      __builtin_memcpy(&v1, y, 16);
      *reinterpret_cast<u32x4*>(dst + i0) = v0;
      *reinterpret_cast<u32x4*>(dst + i1) = v1;
    } else {
      for (int p = p0; p < min(p0 + V, a.half); ++p) {
        const int i0 = a.interleaved ? 2 * p : p, i1 = a.interleaved ? 2 * p + 1 : a.half + p;
        const float x0 = E::get(src[i0]), y0 = E::get(src[i1]);
        dst[i0] = E::put(x0 * cs[p] - y0 * sn[p]);
        dst[i1] = E::put(y0 * cs[p] + x0 * sn[p]);
      }
    }
  }
  if (PAGED && cached) {
    const int pieces = a.D / V;
    for (int u = blockIdx.y * kRotThreads + tid; u < v_rows * pieces; u += gridDim.y * kRotThreads) {
      const size_t e0 = (size_t)u * V;
      *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.V) + cache_row + e0) =
          *reinterpret_cast<const u32x4*>(static_cast<const T*>(a.V) + (size_t)t * a.Hkv * a.D + e0);
    }
    if (a.c.W && blockIdx.y == 0 && tid < a.Hkv)
      a.c.W[((size_t)page * a.Hkv + tid) * (1 << a.c.shift) + slot] = a.mask && a.mask[t] ? INFINITY : 0.f;
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  const dim3 grid(a.total, 1), block(kRotThreads);
  if (a.r.B > 0) {
    if (dtype == SEKA_BF16) hipLaunchKernelGGL((rotary_kernel<uint16_t, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<float, true>), grid, block, 0, s, a);
  } else {
    if (dtype == SEKA_BF16) hipLaunchKernelGGL((rotary_kernel<uint16_t, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rotary_kernel<float, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace seka
