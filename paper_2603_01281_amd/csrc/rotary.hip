// Rotary positions, and their use where new tokens enter a cache of pages.
//
// A pair (x, y) of a head's first 2 half elements at position p turns by p f_i:  (x cos - y sin, y cos + x sin), times a factor.
// f_i p is formed in revolutions in 64 bits and its whole part dropped there: at position 10^6 the angle of the fastest pair in
// 32 bits would be off by 0.03 radians.
//
// HBM-bound: every row is read and written once.  A workgroup takes one token (grid.y: a share of its heads); one sine and cosine
// per pair, which all heads of the token share, go through LDS while the first rows are on their way.  A thread owns whole pairs
// (16 bytes on each side), so input and output may be the same memory.
// 16381 tokens, 32 + 8 heads of 128, half of each turned: 335 MB in 64 us, 5.2 TB/s, what a large copy reaches; 48 tokens: 3.6 us of a call's 6.6.
// Into pages, fp32, 4460 tokens: 219 MB in 50 us, 4.4 TB/s (one unit per thread and workgroups for all of them: 60); 64 requests at one token: 4.9 us of a call's 7.
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

// Work of a token in units: V pairs of a row of Q or K, or V elements that are copied (behind the rotated part; V in the paged form).
template <typename T, bool PAGED>
struct RotUnit {
  static constexpr int V = RotElem<T>::V;
  enum Kind { PAIRS, PAIRS_BY_ELEMENT, COPY, COPY_BY_ELEMENT };
  Kind kind;
  bool is_q, is_v;
  int h, i0, i1, n;      // head; first elements; pairs or elements

  // What every thread would work out again for each of its units; u / per_row is the upper half of u times `inverse`, exact below u per_row = 2^32
  // (0: a division).
  struct Row {
    int nrot, per_row, turned;
    uint32_t inverse;
    __device__ __forceinline__ Row(const RotaryArgs& a) {
      nrot = (a.half + V - 1) / V;
      per_row = nrot + (a.D - 2 * a.half + V - 1) / V;
      turned = ((a.Q ? a.Hq : 0) + (a.K ? a.Hkv : 0)) * per_row;
      inverse = per_row == 1 || (uint32_t)turned > 0xffffffffu / (uint32_t)per_row ? 0 : 0xffffffffu / (uint32_t)per_row + 1u;
    }
  };

  __device__ __forceinline__ RotUnit(const RotaryArgs& a, const Row& r, int u) {
    const int dim = 2 * a.half, nrot = r.nrot, per_row = r.per_row, q_rows = a.Q ? a.Hq : 0;
    is_v = PAGED && u >= r.turned;
    if (is_v) {                              // of all heads' values in a row
      is_q = false;
      h = 0;
      i0 = i1 = (u - r.turned) * V;
      n = V;
      kind = COPY;
      return;
    }
    const int row = r.inverse ? (int)__umulhi((uint32_t)u, r.inverse) : u / per_row, part = u - row * per_row;
    is_q = row < q_rows;
    h = is_q ? row : row - q_rows;
    if (part >= nrot) {
      i0 = i1 = dim + (part - nrot) * V;
      n = min(V, a.D - i0);
      kind = dim % V == 0 ? COPY : COPY_BY_ELEMENT;
    } else {
      const int p0 = part * V;
      n = min(V, a.half - p0);
      i0 = a.interleaved ? 2 * p0 : p0;
      i1 = a.interleaved ? 2 * p0 + V : a.half + p0;
      kind = n == V && (a.interleaved || a.half % V == 0) ? PAIRS : PAIRS_BY_ELEMENT;
    }
  }
  __device__ __forceinline__ const T* source(const RotaryArgs& a, int t) const {
    const void* x = is_v ? a.V : is_q ? a.Q : a.K;
    return static_cast<const T*>(x) + ((size_t)t * (is_q ? a.Hq : a.Hkv) + h) * a.D;
  }
};

template <typename T, bool PAGED>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  using E = RotElem<T>;
  using Unit = RotUnit<T, PAGED>;
  constexpr int V = E::V;
  __shared__ float cs[64], sn[64];
  const int t = blockIdx.x, tid = threadIdx.x;
  const typename Unit::Row per(a);
  const int units = per.turned + (PAGED ? a.Hkv * (a.D / V) : 0), stride = gridDim.y * kRotThreads;

  // the first unit's loads are on their way while the token's place and its angles are found
  int u = blockIdx.y * kRotThreads + tid;
  Unit x(a, per, min(u, units - 1));
  u32x4 v0 = {0, 0, 0, 0}, v1 = {0, 0, 0, 0};
  auto load = [&]() __attribute__((always_inline)) {
    const T* src = x.source(a, t);
    if (x.kind == Unit::PAIRS || x.kind == Unit::COPY) v0 = *reinterpret_cast<const u32x4*>(src + x.i0);
    if (x.kind == Unit::PAIRS) v1 = *reinterpret_cast<const u32x4*>(src + x.i1);
  };
  if (u < units) load();

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
  while (u < units) {
    const T* src = x.source(a, t);
    T* dst = x.is_q ? static_cast<T*>(a.Q_out) + ((size_t)t * a.Hq + x.h) * a.D
             : PAGED ? static_cast<T*>(x.is_v ? a.c.V : a.c.K) + cache_row + (size_t)x.h * a.D
                     : static_cast<T*>(a.K_out) + ((size_t)t * a.Hkv + x.h) * a.D;
    const int p0 = a.interleaved ? x.i0 / 2 : x.i0;
    if (PAGED && !x.is_q && !cached) {
      // a token that has no place in the cache
    } else if (x.kind == Unit::PAIRS) {
      T p[V], q[V];
      __builtin_memcpy(p, &v0, 16);
      __builtin_memcpy(q, &v1, 16);
      if (a.interleaved) {
#pragma unroll
        for (int k = 0; k < V; k += 2) {
          const int i = p0 + k / 2, j = i + V / 2;
          const float x0 = E::get(p[k]), x1 = E::get(p[k + 1]), y0 = E::get(q[k]), y1 = E::get(q[k + 1]);
          p[k] = E::put(x0 * cs[i] - x1 * sn[i]);
          p[k + 1] = E::put(x1 * cs[i] + x0 * sn[i]);
          q[k] = E::put(y0 * cs[j] - y1 * sn[j]);
          q[k + 1] = E::put(y1 * cs[j] + y0 * sn[j]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float x0 = E::get(p[k]), y0 = E::get(q[k]);
          p[k] = E::put(x0 * cs[p0 + k] - y0 * sn[p0 + k]);
          q[k] = E::put(y0 * cs[p0 + k] + x0 * sn[p0 + k]);
        }
      }
      __builtin_memcpy(&v0, p, 16);
      __builtin_memcpy(&v1, q, 16);
      *reinterpret_cast<u32x4*>(dst + x.i0) = v0;
      *reinterpret_cast<u32x4*>(dst + x.i1) = v1;
    } else if (x.kind == Unit::COPY) {
      if (src != dst) *reinterpret_cast<u32x4*>(dst + x.i0) = v0;
    } else if (x.kind == Unit::COPY_BY_ELEMENT) {
      if (src != dst)
        for (int e = 0; e < x.n; ++e) dst[x.i0 + e] = src[x.i0 + e];
    } else {
      for (int k = 0; k < x.n; ++k) {
        const int e0 = a.interleaved ? x.i0 + 2 * k : x.i0 + k, e1 = a.interleaved ? e0 + 1 : x.i1 + k;
        const float x0 = E::get(src[e0]), y0 = E::get(src[e1]);
        dst[e0] = E::put(x0 * cs[p0 + k] - y0 * sn[p0 + k]);
        dst[e1] = E::put(y0 * cs[p0 + k] + x0 * sn[p0 + k]);
      }
    }
    u += stride;
    if (u < units) {
      x = Unit(a, per, u);
      load();
    }
  }
  if (PAGED && cached && a.c.W && blockIdx.y == 0 && tid < a.Hkv)
    a.c.W[((size_t)page * a.Hkv + tid) * (1 << a.c.shift) + slot] = a.mask && a.mask[t] ? INFINITY : 0.f;
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  // a workgroup per token, and where those are few so many that every thread has one unit: the rest is waiting for memory
  const int row_units = (a.D + 15) / 16 * (dtype == SEKA_BF16 ? 1 : 2) + 1;
  const int units = ((a.Q ? a.Hq : 0) + 2 * (a.K ? a.Hkv : 0)) * row_units;
  const int most = std::max(1, (units + kRotThreads - 1) / kRotThreads);
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
