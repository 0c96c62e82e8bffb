// Rotary positions, and their use where new tokens enter a cache of pages.
//
// A pair (x, y) of a head's first 2 half elements at position p turns by p f_i:  (x cos - y sin, y cos + x sin), times a factor.
// f_i p is formed in revolutions in 64 bits and its whole part dropped there: at position 10^6 the angle of the fastest pair in
// 32 bits would be off by 0.03 radians.
//
// HBM-bound: every row is read and written once.  A workgroup takes one token (grid.y: a share of its heads); one sine and cosine
// per pair, which all heads of the token share, go through LDS while the first rows are on their way.  A thread owns whole pairs
// (16 bytes on each side), the same ones of every row that it takes, so input and output may be the same memory, and finds its place in a row once
// (a unit's place found by division each time, which is as much work as turning it: 4460 tokens into pages, fp32, 49.8 us).
// 16381 tokens, 32 + 8 heads of 128, half of each turned: 335 MB in 64 us, 5.2 TB/s, what a large copy reaches; 48 tokens: 3.6 us of a call's 6.6.
// Into pages, fp32, 4460 tokens: 219 MB in 47.4 us, 4.6 TB/s; 64 requests at one token: 4.9 us of a call's 7.
#include <algorithm>

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

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

template <typename T, bool PAGED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  using E = RotElem<T>;
  constexpr int V = E::V;
  enum Kind { PAIRS, PAIRS_BY_ELEMENT, COPY, COPY_BY_ELEMENT };
  __shared__ float cs[64], sn[64];
  const int t = blockIdx.x, tid = threadIdx.x;

  // This thread's part of every row that it takes: V pairs, or V elements behind the rotated ones.
  const int dim = 2 * a.half, nrot = (a.half + V - 1) / V, per_row = nrot + (a.D - dim + V - 1) / V, step = kRotThreads / per_row;
  const int part = tid % per_row, q_rows = a.Q ? a.Hq : 0, rows = q_rows + (a.K ? a.Hkv : 0);
  const bool turns = part < nrot;
  const int p0 = part * V;                   // its first pair
  const int i0 = !turns ? dim + (part - nrot) * V : a.interleaved ? 2 * p0 : p0, i1 = !turns ? i0 : a.interleaved ? 2 * p0 + V : a.half + p0;
  const int n = turns ? min(V, a.half - p0) : min(V, a.D - i0);                  // pairs or elements
  const Kind kind = turns ? (n == V && (a.interleaved || a.half % V == 0) ? PAIRS : PAIRS_BY_ELEMENT) : dim % V == 0 ? COPY : COPY_BY_ELEMENT;
  int row = tid < step * per_row ? blockIdx.y * step + tid / per_row : rows;     // the next one: + step gridDim.y
  const int v_pieces = PAGED ? a.Hkv * (a.D / V) : 0;                            // of all heads' values
  int piece = blockIdx.y * kRotThreads + tid;
  auto source = [&](int row) __attribute__((always_inline)) -> const T* {
    return row < q_rows ? static_cast<const T*>(a.Q) + ((size_t)t * a.Hq + row) * a.D : static_cast<const T*>(a.K) + ((size_t)t * a.Hkv + (row - q_rows)) * a.D;
  };
  // the first loads are on their way while the token's place and its angles are found
  u32x4 v0 = {0, 0, 0, 0}, v1 = {0, 0, 0, 0}, w = {0, 0, 0, 0};
  auto load = [&]() __attribute__((always_inline)) {
    const T* src = source(row);
    if (kind == PAIRS || kind == COPY) v0 = *reinterpret_cast<const u32x4*>(src + i0);
    if (kind == PAIRS) v1 = *reinterpret_cast<const u32x4*>(src + i1);
  };
  auto load_v = [&]() __attribute__((always_inline)) { w = *reinterpret_cast<const u32x4*>(static_cast<const T*>(a.V) + (size_t)t * a.Hkv * a.D + (size_t)piece * V); };
  if (row < rows) load();
  if (PAGED && piece < v_pieces) load_v();

  // ---- where the token lies ----
  bool cached = false;
  int slot = 0, page = 0, pos = 0;
  if (PAGED) {
    // the request is the number of requests that end at or before row t
    int b = 0;
    for (int b0 = 0; b0 < a.r.B; b0 += kRotThreads)
      b += __syncthreads_count(b0 + tid < a.r.B && a.r.cu[min(b0 + tid, a.r.B - 1) + 1] <= t);
    if (b >= a.r.B) return;                  // the same in every thread
    const ChunkExtent e = chunk_extent(a.r, a.c, b);
    const int i = t - e.row0, j = e.len - e.n + i;
    if (i < 0 || i >= e.n) return;
    cached = j >= 0;
    if (cached) {
      page = page_of(a.c, b, j);
      slot = j & ((1 << a.c.shift) - 1);
    }
    pos = j;
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

  const size_t cache_row = ((((size_t)page << a.c.shift) + slot) * a.Hkv) * a.D;
  auto target = [&](int row) __attribute__((always_inline)) -> T* {
    if (row < q_rows) return static_cast<T*>(a.Q_out) + ((size_t)t * a.Hq + row) * a.D;
    return PAGED ? static_cast<T*>(a.c.K) + cache_row + (size_t)(row - q_rows) * a.D : static_cast<T*>(a.K_out) + ((size_t)t * a.Hkv + (row - q_rows)) * a.D;
  };
  while (row < rows) {
    if (sizeof(T) == 2) asm volatile("" ::: "memory");     // sixteen angles in registers would halve the waves: they are read from LDS for each row
    const T* src = source(row);
    T* dst = target(row);
    if (PAGED && row >= q_rows && !cached) {
      // a token that has no place in the cache
    } else if (kind == PAIRS) {
      T p[V], q[V];
      float c[V], s[V];                      // of its pairs, the same in every row
#pragma unroll
      for (int k = 0; k < V; ++k) {
        c[k] = cs[p0 + k];
        s[k] = sn[p0 + k];
      }
      __builtin_memcpy(p, &v0, 16);
      __builtin_memcpy(q, &v1, 16);
      if (a.interleaved) {
#pragma unroll
        for (int k = 0; k < V; k += 2) {
          const int i = k / 2, j = i + V / 2;
          const float x0 = E::get(p[k]), x1 = E::get(p[k + 1]), y0 = E::get(q[k]), y1 = E::get(q[k + 1]);
          p[k] = E::put(x0 * c[i] - x1 * s[i]);
          p[k + 1] = E::put(x1 * c[i] + x0 * s[i]);
          q[k] = E::put(y0 * c[j] - y1 * s[j]);
          q[k + 1] = E::put(y1 * c[j] + y0 * s[j]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float x0 = E::get(p[k]), y0 = E::get(q[k]);
          p[k] = E::put(x0 * c[k] - y0 * s[k]);
          q[k] = E::put(y0 * c[k] + x0 * s[k]);
        }
      }
      __builtin_memcpy(&v0, p, 16);
      __builtin_memcpy(&v1, q, 16);
      *reinterpret_cast<u32x4*>(dst + i0) = v0;
      *reinterpret_cast<u32x4*>(dst + i1) = v1;
    } else if (kind == COPY) {
      if (src != dst) *reinterpret_cast<u32x4*>(dst + i0) = v0;
    } else if (kind == COPY_BY_ELEMENT) {
      if (src != dst)
        for (int e = 0; e < n; ++e) dst[i0 + e] = src[i0 + e];
    } else {
      for (int k = 0; k < n; ++k) {
        const int e0 = a.interleaved ? i0 + 2 * k : i0 + k, e1 = a.interleaved ? e0 + 1 : i1 + k;
        const float x0 = E::get(src[e0]), y0 = E::get(src[e1]);
        dst[e0] = E::put(x0 * cs[p0 + k] - y0 * sn[p0 + k]);
        dst[e1] = E::put(y0 * cs[p0 + k] + x0 * sn[p0 + k]);
      }
    }
    row += step * gridDim.y;
    if (row < rows) load();
  }
  while (PAGED && cached && piece < v_pieces) {
    *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.V) + cache_row + (size_t)piece * V) = w;
    piece += kRotThreads * gridDim.y;
    if (piece < v_pieces) load_v();
  }
  if (PAGED && cached && a.c.W && blockIdx.y == 0 && tid < a.Hkv)
    a.c.W[((size_t)page * a.Hkv + tid) * (1 << a.c.shift) + slot] = a.mask && a.mask[t] ? INFINITY : 0.f;
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  // a workgroup per token, and where those are few so many that every thread has one unit: the rest is waiting for memory
  const int V = dtype == SEKA_BF16 ? 8 : 4, per_row = (a.half + V - 1) / V + (a.D - 2 * a.half + V - 1) / V, step = kRotThreads / per_row;
  const int rows = (a.Q ? a.Hq : 0) + (a.K ? a.Hkv : 0);
  const int most = std::max(1, (rows + step - 1) / step);
  const dim3 grid(a.total, std::min(most, std::max(1, 1024 / a.total))), block(kRotThreads);
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
