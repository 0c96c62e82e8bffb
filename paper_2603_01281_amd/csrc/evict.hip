// seka_cache_evict: a cache is cut to `budget` tokens per KV head: the last `recent` ones and, of the others, those with the
// largest accumulated attention weight, ties to the earlier token.  What stays keeps its order.
//
// 1. evict_select_kernel, one workgroup per (request, KV head): the weights become ordered integers in LDS; the (budget - recent)-th
//    largest is found by four rounds of 256 counters over its bytes; waves then write down the places of what stays, each
//    over its own part of the tokens, with ranks from ballots.
// 2. evict_move_kernel: rows of K and V (and the weights) to their new places.  A row moves to an earlier place or stays, so within
//    one pool a workgroup passes the rows in order, reads a block of rows, waits for all its waves and writes it: no source is
//    overwritten before it was read.  Between two pools the rows are independent and workgroups share them.
#include <algorithm>

#include "paged.h"

namespace seka {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelCopies = 16;                  // of every counter: lanes that count the same byte meet in one of them
constexpr int kSelKeys = 30 * 1024;             // tokens whose keys LDS holds
constexpr int kMoveThreads = 256, kMoveRows = 4;     // rows of a thread whose pieces are in flight together

// Larger weights have larger keys; both zeros the same one; what is not a number the smallest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? (u == 0x80000000u ? 0x80000000u : ~u) : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t keys[];            // [min(candidates, kSelKeys)]
  __shared__ __attribute__((aligned(16))) uint32_t hist[2][256 * kSelCopies];
  __shared__ __attribute__((aligned(16))) uint32_t total[2][256];
  __shared__ int sm_gt[kSelWaves], sm_eq[kSelWaves];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.src.lens[b], 0), a.src.cap);
  int* kept = a.kept + ((size_t)b * a.Hkv + h) * a.budget;
  if (n <= a.budget) {
    for (int k = tid; k < a.budget; k += kSelThreads) kept[k] = k < n ? k : -1;
    return;
  }
  const int m = n - a.recent;                   // candidates
  const int want = a.budget - a.recent;         // of them; < m
  for (int k = tid; k < a.recent; k += kSelThreads) kept[want + k] = m + k;
  if (want == 0) return;
  const int shift = a.src.shift;
  const bool held = m <= kSelKeys;
  auto weight_at = [&](int j) __attribute__((always_inline)) -> float {
    return a.src.W[(((size_t)page_of(a.src, b, j) * a.Hkv + h) << shift) + (j & ((1 << shift) - 1))];
  };
  auto key_at = [&](int j) __attribute__((always_inline)) -> uint32_t { return held ? keys[j] : weight_key(weight_at(j)); };
  if (held) {
    constexpr int U = 8;                        // tokens of a thread whose loads are in flight together
    for (int j0 = tid; j0 < m; j0 += U * kSelThreads) {
      float w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = weight_at(min(j0 + u * kSelThreads, m - 1));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j0 + u * kSelThreads < m) keys[j0 + u * kSelThreads] = weight_key(w[u]);
    }
  }
  for (int k = tid; k < 256 * kSelCopies; k += kSelThreads) hist[0][k] = 0;
  __syncthreads();
  // ---- the want-th largest key, a byte at a time ----
  uint32_t prefix = 0;
  int need = want;                              // of the keys that begin with prefix
  for (int byte = 3; byte >= 0; --byte) {
    const int now = byte & 1 ? 0 : 1;           // counters of this byte; the others are cleared for the next one
#pragma unroll 4
    for (int j = tid; j < m; j += kSelThreads) {
      const uint32_t u = key_at(j);
      if (byte == 3 || (u >> (8 * byte + 8)) == prefix) atomicAdd(&hist[now][((u >> (8 * byte)) & 255) * kSelCopies + (lane & (kSelCopies - 1))], 1u);
    }
    __syncthreads();
    {                                           // four threads to a counter, four copies each
      uint32_t c = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) c += hist[now][4 * tid + k];
      c += __shfl_xor(c, 1);
      c += __shfl_xor(c, 2);
      if ((tid & 3) == 0) total[now][tid >> 2] = c;
#pragma unroll
      for (int k = 0; k < 4; ++k) hist[now ^ 1][4 * tid + k] = 0;
    }
    __syncthreads();
    // every wave finds the byte by itself; lane l: the bytes 255 - 4 l .. 252 - 4 l, the largest first
    uint32_t c[4], mine = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) mine += c[x] = total[now][255 - 4 * lane - x];
    uint32_t above = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(above, d);
      if (lane >= d) above += o;
    }
    const unsigned long long hit = __ballot((int)above >= need);       // the first lane that reaches it
    const int at = __builtin_ctzll(hit);
    above = __shfl(above - mine, at);
    uint32_t digit = 255 - 4 * at;
#pragma unroll
    for (int x = 0; x < 3; ++x) {
      const uint32_t cx = __shfl(c[x], at);
      if (digit == 255u - 4 * at - x && (int)(above + cx) < need) {
        above += cx;
        --digit;
      }
    }
    prefix = prefix << 8 | digit;
    need -= (int)above;
  }
  // ---- every key above prefix, and the first `need` that equal it, in order ----
  const int per = ((m + kSelWaves - 1) / kSelWaves + 63) / 64 * 64;
  const int j0 = min(wave * per, m), j1 = min(j0 + per, m);
  int gt = 0, eq = 0;
  for (int j = j0 + lane; j < j0 + per; j += 64) {
    const uint32_t u = j < j1 ? key_at(j) : 0u;
    gt += __popcll(__ballot(j < j1 && u > prefix));
    eq += __popcll(__ballot(j < j1 && u == prefix));
  }
  if (lane == 0) {
    sm_gt[wave] = gt;
    sm_eq[wave] = eq;
  }
  __syncthreads();
  int gt0 = 0, eq0 = 0;
  for (int w = 0; w < wave; ++w) {
    gt0 += sm_gt[w];
    eq0 += sm_eq[w];
  }
  for (int j = j0 + lane; j < j0 + per; j += 64) {
    const uint32_t u = j < j1 ? key_at(j) : 0u;
    const unsigned long long g = __ballot(j < j1 && u > prefix), q = __ballot(j < j1 && u == prefix);
    const unsigned long long below = (1ull << lane) - 1;
    const int my_eq = eq0 + __popcll(q & below), my_gt = gt0 + __popcll(g & below);
    const bool is_gt = (g >> lane) & 1, is_eq = (q >> lane) & 1;
    if (is_gt || (is_eq && my_eq < need)) kept[my_gt + min(my_eq, need)] = j;
    gt0 += __popcll(g);
    eq0 += __popcll(q);
  }
}

// blockIdx: x: KV head (the heads of a token lie side by side), y: part of the work, z: request.  IN_ORDER: y = 0 .. 2 * parts - 1 are the
// column parts of K and V, 2 * parts the weights; otherwise y takes a share of the rows with everything that belongs to them.
template <bool IN_ORDER>
__global__ __launch_bounds__(IN_ORDER ? 1024 : kMoveThreads) void evict_move_kernel(EvictArgs a, int parts) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  const int h = blockIdx.x, part = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int n = min(max(a.src.lens[b], 0), a.src.cap), m = min(min(n, a.budget), a.dst.cap);
  if (part == 0 && h == 0 && tid == 0) a.lens_out[b] = m;
  const int* kept = a.kept + ((size_t)b * a.Hkv + h) * a.budget;
  const int s_slots = (1 << a.src.shift) - 1, d_slots = (1 << a.dst.shift) - 1;
  auto from = [&](int j) __attribute__((always_inline)) -> size_t { return ((((size_t)page_of(a.src, b, j)) << a.src.shift) + (j & s_slots)) * a.Hkv + h; };
  auto to = [&](int k) __attribute__((always_inline)) -> size_t { return ((((size_t)page_of(a.dst, b, k)) << a.dst.shift) + (k & d_slots)) * a.Hkv + h; };
  auto w_from = [&](int j) __attribute__((always_inline)) -> size_t { return (((size_t)page_of(a.src, b, j) * a.Hkv + h) << a.src.shift) + (j & s_slots); };
  auto w_to = [&](int k) __attribute__((always_inline)) -> size_t { return (((size_t)page_of(a.dst, b, k) * a.Hkv + h) << a.dst.shift) + (k & d_slots); };
  if (IN_ORDER) {
    constexpr int NT = 1024;
    if (part == 2 * parts) {
      for (int k0 = 0; k0 < m; k0 += NT) {
        const int k = k0 + tid;
        const float w = k < m ? a.src.W[w_from(kept[k])] : 0.f;
        __syncthreads();
        if (k < m) a.dst.W[w_to(k)] = w;
      }
      return;
    }
    const int pieces = a.row_bytes / 16 / parts;          // 16-byte pieces of a row that this workgroup moves
    const int rows = NT / pieces;
    const bool is_v = part >= parts;
    const char* src = static_cast<const char*>(is_v ? a.src.V : a.src.K);
    char* dst = static_cast<char*>(is_v ? a.dst.V : a.dst.K);
    const size_t off = 16 * ((part % parts) * pieces + tid % pieces);
    for (int k0 = 0; k0 < m; k0 += rows) {
      const int k = k0 + tid / pieces;
      u32x4 v = {0, 0, 0, 0};
      if (k < m) v = *reinterpret_cast<const u32x4*>(src + from(kept[k]) * a.row_bytes + off);
      __syncthreads();
      if (k < m) *reinterpret_cast<u32x4*>(dst + to(k) * a.row_bytes + off) = v;
    }
  } else {
    constexpr int U = kMoveRows;
    const int pieces = a.row_bytes / 16, rows = kMoveThreads / pieces;
    const size_t off = 16 * (tid % pieces);
    for (int k0 = part * rows * U + tid / pieces; k0 < m; k0 += gridDim.y * rows * U) {
      u32x4 x[U], y[U];
      int j[U];
      size_t d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) j[u] = kept[min(k0 + u * rows, m - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u) d[u] = to(min(k0 + u * rows, m - 1)) * a.row_bytes + off;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t s0 = from(j[u]) * a.row_bytes + off;
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const char*>(a.src.K) + s0));
        y[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const char*>(a.src.V) + s0));
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u * rows < m) {
          __builtin_nontemporal_store(x[u], reinterpret_cast<u32x4*>(static_cast<char*>(a.dst.K) + d[u]));
          __builtin_nontemporal_store(y[u], reinterpret_cast<u32x4*>(static_cast<char*>(a.dst.V) + d[u]));
        }
    }
    // the weights, one per thread
    for (int k = part * kMoveThreads + tid; k < m; k += gridDim.y * kMoveThreads) a.dst.W[w_to(k)] = a.src.W[w_from(kept[k])];
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  const int most = std::min(std::max(a.src.cap - a.recent, 1), kSelKeys);
  const size_t smem = (size_t)most * sizeof(uint32_t);
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(evict_select_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_select_kernel, dim3(a.Hkv, a.B), dim3(kSelThreads), smem, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.dst.K == a.src.K) {
    const int parts = a.row_bytes / 64;                   // pieces of 64 bytes
    hipLaunchKernelGGL((evict_move_kernel<true>), dim3(a.Hkv, 2 * parts + 1, a.B), dim3(1024), 0, s, a, parts);
  } else {
    const int rows = kMoveThreads / (a.row_bytes / 16) * kMoveRows, most_rows = std::min(a.budget, a.src.cap);
    const int share = std::max(1, std::min((most_rows + rows - 1) / rows, 4096 / std::max(1, a.Hkv * a.B)));
    hipLaunchKernelGGL((evict_move_kernel<false>), dim3(a.Hkv, share, a.B), dim3(kMoveThreads), 0, s, a, 1);
  }
  return hipGetLastError();
}

}  // namespace seka
