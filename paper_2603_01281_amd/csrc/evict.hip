// seka_cache_evict: a cache is cut to `budget` tokens per KV head: the last `recent` ones and, of the others, those with the
// largest accumulated attention weight, ties to the earlier token.  What stays keeps its order.
//
// 1. evict_select_kernel, one workgroup per (request, KV head): the weights become ordered integers in LDS; the (budget - recent)-th
//    largest is found by four rounds of 256 counters over its bytes; waves then write down the places of what stays, each
//    over its own part of the tokens, with ranks from ballots.  Up to kSelFew candidates count the others that come before them instead.
// 2. evict_move_kernel: rows of K and V (and the weights) to their new places.  A row moves to an earlier place or stays, so within
//    one pool a workgroup passes the rows in order, reads a block of rows, waits for all its waves and writes it: no source is
//    overwritten before it was read.  Between two pools the rows are independent and workgroups share them.
// 16 requests of 16384, 8 heads of 128, cut to 4096: 108 us: 19 for the selection (the histogram's rounds; 8 MB of weights) and 85 for 413 MB
// of rows of 256 bytes from anywhere, 4.9 TB/s.  One request of 4097: 14.4 us, of them 10.4 the selection's chain of four rounds.
#include <algorithm>

#include "paged.h"

namespace seka {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelCopies = 16;                  // of every counter: lanes that count the same byte meet in one of them
constexpr int kSelKeys = 30 * 1024;             // tokens whose keys LDS holds
constexpr int kSelFew = 256;                    // candidates that are ranked by counting (3 requests of up to 207, a call: 9.0 us, in rounds 11.5)
constexpr int kMoveThreads = 256, kMoveRows = 4;     // rows of a thread whose pieces are in flight together

// Larger weights have larger keys; both zeros the same one; what is not a number the smallest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? (u == 0x80000000u ? 0x80000000u : ~u) : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];            // [min(candidates, kSelKeys), whole quads]
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
  // tokens four at a time: a page has eight or more
  const int shift = a.src.shift, quads = (m + 3) / 4;
  const bool held = m <= kSelKeys;
  auto weights_of = [&](int q) __attribute__((always_inline)) -> f32x4 {
    const int j = 4 * q;
    return *reinterpret_cast<const f32x4*>(a.src.W + (((size_t)page_of(a.src, b, j) * a.Hkv + h) << shift) + (j & ((1 << shift) - 1)));
  };
  auto keys_of = [&](f32x4 w) __attribute__((always_inline)) -> u32x4 {
    u32x4 k;
#pragma unroll
    for (int x = 0; x < 4; ++x) k[x] = weight_key(w[x]);
    return k;
  };
  u32x4* const keys4 = reinterpret_cast<u32x4*>(keys);
  auto keys_at = [&](int q) __attribute__((always_inline)) -> u32x4 { return held ? keys4[q] : keys_of(weights_of(q)); };
  if (held) {
    constexpr int U = 4;                        // quads of a thread whose loads are in flight together
    for (int q0 = tid; q0 < quads; q0 += U * kSelThreads) {
      f32x4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = weights_of(min(q0 + u * kSelThreads, quads - 1));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (q0 + u * kSelThreads < quads) keys4[q0 + u * kSelThreads] = keys_of(w[u]);
    }
  }
  if (m <= kSelFew) {                           // four threads to a candidate, a quarter of the others each
    __syncthreads();
    if (tid < 4 * quads - m) keys[m + tid] = 0;                // what is behind the candidates comes before none of them
    __syncthreads();
    const int j = tid >> 2;
    const uint32_t mine = j < m ? keys[j] : 0xffffffffu;
    int before = 0;                             // keys that come before its own
#pragma unroll 4
    for (int q = tid & 3; q < quads; q += 4) {
      const u32x4 u = keys4[q];
#pragma unroll
      for (int x = 0; x < 4; ++x) before += (int)(u[x] > mine) + (int)((u[x] == mine) & (4 * q + x < j));
    }
    before += __shfl_xor(before, 1);
    before += __shfl_xor(before, 2);
    const bool stays = j < m && before < want;
    const unsigned long long all = __ballot(stays && (tid & 3) == 0);
    if (lane == 0) sm_gt[wave] = __popcll(all);
    __syncthreads();
    int at = __popcll(all & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) at += sm_gt[w];
    if (stays && (tid & 3) == 0) kept[at] = j;
    return;
  }
  for (int k = tid; k < 256 * kSelCopies; k += kSelThreads) hist[0][k] = 0;
  __syncthreads();
  // ---- the want-th largest key, a byte at a time ----
  uint32_t prefix = 0;
  int need = want;                              // of the keys that begin with prefix
  for (int byte = 3; byte >= 0; --byte) {
    const int now = byte & 1 ? 0 : 1;           // counters of this byte; the others are cleared for the next one
    for (int q = tid; q < quads; q += kSelThreads) {
      const u32x4 u = keys_at(q);
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (4 * q + x < m && (byte == 3 || (u[x] >> (8 * byte + 8)) == prefix))
          atomicAdd(&hist[now][((u[x] >> (8 * byte)) & 255) * kSelCopies + (lane & (kSelCopies - 1))], 1u);
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
  // ---- every key above prefix, and the first `need` that equal it, in order: a wave takes consecutive quads, a lane one ----
  const int per = ((quads + kSelWaves - 1) / kSelWaves + 63) / 64 * 64;
  const int q0 = wave * per, q1 = min(q0 + per, quads);
  // how many of the quad are above and equal
  auto count = [&](int q, u32x4& u, int& gt, int& eq) __attribute__((always_inline)) {
    gt = eq = 0;
    u = u32x4{0, 0, 0, 0};
    if (q < q1) {
      u = keys_at(q);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        gt += 4 * q + x < m && u[x] > prefix;
        eq += 4 * q + x < m && u[x] == prefix;
      }
    }
  };
  // sum over the lanes selected, of numbers of 0 .. 4
  auto over = [&](int v, unsigned long long lanes) __attribute__((always_inline)) -> int {
    return __popcll(__ballot(v & 1) & lanes) + 2 * __popcll(__ballot(v & 2) & lanes) + 4 * __popcll(__ballot(v & 4) & lanes);
  };
  int gt_all = 0, eq_all = 0;
  for (int q = q0 + lane; q < q0 + per; q += 64) {
    u32x4 u;
    int gt, eq;
    count(q, u, gt, eq);
    gt_all += over(gt, ~0ull);
    eq_all += over(eq, ~0ull);
  }
  if (lane == 0) {
    sm_gt[wave] = gt_all;
    sm_eq[wave] = eq_all;
  }
  __syncthreads();
  int gt0 = 0, eq0 = 0;
  for (int w = 0; w < wave; ++w) {
    gt0 += sm_gt[w];
    eq0 += sm_eq[w];
  }
  for (int q = q0 + lane; q < q0 + per; q += 64) {
    u32x4 u;
    int gt, eq;
    count(q, u, gt, eq);
    const unsigned long long below = (1ull << lane) - 1;
    int my_gt = gt0 + over(gt, below), my_eq = eq0 + over(eq, below);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const bool is_gt = q < q1 && 4 * q + x < m && u[x] > prefix, is_eq = q < q1 && 4 * q + x < m && u[x] == prefix;
      if (is_gt || (is_eq && my_eq < need)) kept[my_gt + min(my_eq, need)] = 4 * q + x;
      my_gt += is_gt;
      my_eq += is_eq;
    }
    gt0 += over(gt, ~0ull);
    eq0 += over(eq, ~0ull);
  }
}

// blockIdx: x: KV head (the heads of a token lie side by side), y: part of the work, z: request.  IN_ORDER: y = 0 .. 2 * parts - 1 are the
// column parts of K and V, 2 * parts the weights; otherwise y takes a share of the rows with everything that belongs to them.
template <bool IN_ORDER>
__global__ __launch_bounds__(IN_ORDER ? 1024 : kMoveThreads) void evict_move_kernel(EvictArgs a, int parts) {
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
  const size_t smem = (size_t)(most + 3) / 4 * 16;
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
