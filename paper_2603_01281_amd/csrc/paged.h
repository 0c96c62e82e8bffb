// Caches of pages: what the kernels over them share.
#pragma once
#include "common.h"

namespace seka {

// One pool of pages.  Token j of request b lies in page table[b, j >> shift], at slot j & (page_size - 1).
struct PagedCache {
  void* K;                // dev [num_pages, page_size, Hkv, D]
  void* V;
  float* W;               // dev [num_pages, Hkv, page_size] or nullptr
  const int* table;       // dev [B, max_pages]
  const int* lens;        // dev [B]
  int num_pages, shift, max_pages;
  int cap;                // tokens of a request that a call covers: min(S, max_pages * page_size)
};

// New tokens, packed: request b owns rows cu[b] .. cu[b + 1] - 1 of `total`, the first max_q of them count.
struct ChunkRows {
  const int* cu;          // dev [B + 1]
  int B, total, max_q;
};

struct ChunkExtent {
  int row0, n;            // packed rows of the request's new tokens
  int len;                // cached tokens; new token i is token len - n + i
};

// Whatever cu and lens hold, rows stay in the tensors and tokens in the cache.
__device__ __forceinline__ ChunkExtent chunk_extent(const ChunkRows& r, const PagedCache& c, int b) {
  ChunkExtent e;
  e.row0 = min(max(r.cu[b], 0), r.total);
  e.n = min(max(r.cu[b + 1] - e.row0, 0), min(r.max_q, r.total - e.row0));
  e.len = min(max(c.lens[b], 0), c.cap);
  return e;
}

// Page of token j (0 <= j < cap) of request b: whatever the table holds, a page of the pool.
__device__ __forceinline__ int page_of(const PagedCache& c, int b, int j) {
  return min(max(c.table[(size_t)b * c.max_pages + (j >> c.shift)], 0), c.num_pages - 1);
}

// ---- how the rows and keys of a batch are dealt to workgroups -----------------------------------------------------------
// A request's rows (new token i, head g of the KV head's group: row i G + g) are cut into chunks of R; a chunk's keys are cut
// into `splits` ranges.  All workgroups find their item from the lengths by themselves, in integers, so that every workgroup
// sees the same plan.  T = sum over chunks of their keys (in blocks of 32); a range has about T / slots blocks
// and no fewer than least; slots is a power of two.
struct ChunkPlan {
  int R, G;               // rows per chunk, query heads per KV head; R = 0: one chunk for every request that has cached tokens
  int slots_log2;         // about so many ranges in all, per KV head
  int least;              // blocks of 32 keys in a range, at least
  int max_splits;
  long long streams;      // more blocks than this in all: the keys and values are not kept in the caches
};

struct ChunkItem {
  int b, rc, split, splits;
  bool streams;
  ChunkExtent e;
};

__device__ __forceinline__ int plan_scan(int v) {       // inclusive sum over the wave's lanes
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// The item-th (chunk, range).  Wave-uniform; false: no such item.
__device__ __forceinline__ bool plan_item(const ChunkRows& r, const PagedCache& c, const ChunkPlan& p, int item, ChunkItem& out) {
  const int lane = threadIdx.x & 63;
  ChunkExtent e = {0, 0, 0};
  int chunks = 0, blocks = 0;
  auto look = [&](int b0) __attribute__((always_inline)) {
    chunks = blocks = 0;
    e = ChunkExtent{0, 0, 0};
    if (b0 + lane < r.B) {
      e = chunk_extent(r, c, b0 + lane);
      chunks = p.R ? (int)(((unsigned)e.n * (unsigned)p.G + p.R - 1) / (unsigned)p.R) : e.len > 0;
      blocks = (e.len + 31) >> 5;
    }
  };
  if (r.B == 1) {                        // nothing to add up over requests
    out.b = 0;
    out.e = chunk_extent(r, c, 0);
    chunks = p.R ? (int)(((unsigned)out.e.n * (unsigned)p.G + p.R - 1) / (unsigned)p.R) : out.e.len > 0;
    blocks = (out.e.len + 31) >> 5;
    const unsigned long long T = (unsigned long long)chunks * (unsigned)blocks;
    const unsigned long long per = (T + (1ull << p.slots_log2) - 1) >> p.slots_log2;
    const int L = (int)max((unsigned long long)p.least, min(per, 0x7fffffffull));
    out.streams = T > (unsigned long long)p.streams;
    out.splits = max(1, min((blocks + L - 1) / L, p.max_splits));
    out.rc = item / out.splits;
    out.split = item - out.rc * out.splits;
    return out.rc < chunks;
  }
  unsigned long long T = 0;
  for (int b0 = 0; b0 < r.B; b0 += 64) {
    look(b0);
    unsigned long long w = (unsigned long long)chunks * (unsigned)blocks;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) w += __shfl_xor(w, d);
    T += w;
  }
  out.streams = T > (unsigned long long)p.streams;
  const unsigned long long per = (T + (1ull << p.slots_log2) - 1) >> p.slots_log2;
  const int L = (int)max((unsigned long long)p.least, min(per, 0x7fffffffull));
  int before = 0;                        // items of the requests already passed
  for (int b0 = 0; b0 < r.B; b0 += 64) {
    if (r.B > 64) look(b0);
    const int splits = max(1, min((blocks + L - 1) / L, p.max_splits));
    const int items = chunks * splits, ends = plan_scan(items);
    const int first = before + ends - items;
    const unsigned long long hit = __ballot(item >= first && item < first + items);
    if (hit != 0ull) {
      const int at = __builtin_ctzll(hit);
      const int local = item - __builtin_amdgcn_readlane(first, at);
      const int s = __builtin_amdgcn_readlane(splits, at);
      out.b = b0 + at;
      out.splits = s;
      out.rc = local / s;
      out.split = local % s;
      out.e.row0 = __builtin_amdgcn_readlane(e.row0, at);
      out.e.n = __builtin_amdgcn_readlane(e.n, at);
      out.e.len = __builtin_amdgcn_readlane(e.len, at);
      return true;
    }
    before += __builtin_amdgcn_readlane(ends, 63);
  }
  return false;
}

// Keys that the last row of chunk rc sees, and the range of them that the item takes: whole blocks of 32 but for the last.
__device__ __forceinline__ void plan_range(const ChunkPlan& p, const ChunkItem& it, int& k0, int& k1) {
  const int last_row = min((it.rc + 1) * p.R, it.e.n * p.G) - 1;
  const int seen = p.R ? min(max(it.e.len - it.e.n + last_row / p.G + 1, 0), it.e.len) : it.e.len;
  const int per = (((seen + 31) >> 5) + it.splits - 1) / it.splits * 32;
  k0 = min(it.split * per, seen);
  k1 = min(k0 + per, seen);
}

// Maximum and sum over the four lanes l, l + 16, l + 32, l + 48; the same bits in all of them.
template <typename F>
__device__ __forceinline__ float over_groups(float v, F join) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = join(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return join(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_max(float v) {
  return over_groups(v, [](float x, float y) __attribute__((always_inline)) { return fmaxf(x, y); });
}
__device__ __forceinline__ float groups_sum(float v) {
  return over_groups(v, [](float x, float y) __attribute__((always_inline)) { return x + y; });
}

// Pages of a wave's next blocks of keys, one per lane; NW waves take blocks of KEYS keys in turn.  A page
// that is shorter than a block takes several lanes.
template <int KEYS, int NW>
struct PageWindow {
  int entry;             // this lane's page
  int per_block;         // lanes per block
  int left;              // blocks of the window that are still to come

  __device__ __forceinline__ void load(const PagedCache& c, int b, int key, int k1) {
    const int lane = threadIdx.x & 63;
    const int shift = min(c.shift, __builtin_ctz(KEYS));
    per_block = KEYS >> shift;
    left = 64 / per_block;
    const int j = key + (lane / per_block) * KEYS * NW + ((lane % per_block) << shift);
    entry = page_of(c, b, min(j, k1 - 1));
  }
};

// NT: a load that keeps no place for its line in the caches.
template <bool NT, typename V>
__device__ __forceinline__ V paged_load(const V* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}

struct ChunkArgs {
  const void* Q;
  void* O;
  float* lse;             // dev [Hq, total] or nullptr
  PagedCache c;
  ChunkRows r;
  ChunkPlan p;
  int4* items_of;         // few rows: what the joining kernel has to know of each item
  float* part;            // partial states: [item, Hkv, R, D + 4]: outputs, reference exponent (base 2), sum
  int Hq, Hkv;
  int width;              // long chunks: workgroups per head chunk (chunk_plan.h)
  int4* cuts;             // and where each of them starts: request, block, tile; whether it has no tile there (PipePieces::note)
  float scale;
};

struct RotaryArgs {
  const void* Q;
  void* Q_out;
  const void* K;
  void* K_out;            // dense form; nullptr: K and V go to the pages
  const void* V;
  const uint8_t* mask;
  const int* positions;   // dev [total] or nullptr
  PagedCache c;
  ChunkRows r;            // B = 0: dense form
  int total, S, Hq, Hkv, D;
  int half;               // pairs per head
  int interleaved;
  float factor;
  double turns[64];       // revolutions per position
};

struct WeightsArgs {
  const void* Q;
  const float* lse;       // dev [Hq, total]
  const float* W_in;      // dev [num_pages, Hkv, page_size] or nullptr
  PagedCache c;
  ChunkRows r;
  ChunkPlan p;            // few rows: the ranges of the keys
  int Hq, Hkv, window;
  float scale, decay;
};

struct EvictArgs {
  PagedCache src, dst;
  int* kept;              // dev [B, Hkv, budget]
  int* lens_out;
  int B, Hkv, row_bytes, budget, recent;
};

hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s);
size_t chunk_workspace_bytes(int B, int S, int Hq, int Hkv, int D, int dtype, int total, int max_q);
hipError_t launch_chunk(ChunkArgs a, int D, int dtype, int S, hipStream_t s);
hipError_t launch_weights(const WeightsArgs& a, int D, int dtype, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);

}  // namespace seka
