// How the blocks of query rows of a batch over a cache of pages are dealt to workgroups (chunk_pipe_kernel, chunk_block_f32_kernel).
//
// A request's new tokens are its last n of len cached ones.  Row (p - base) G + g is that of position p and head g of a KV head's group of G,
// with base the multiple of 32 at or before its first new token: 32 positions are G waves of 32 rows, and no wave's rows lie on both sides of
// the end of half a key tile, whatever G.  The waves that have new tokens, WAVES to a block, make up the request's blocks.  (Heads to waves of
// their own, so that a block is 8 / G x 32 positions, left blocks of 256 positions of one head to a group of three.)
// Block k sees the keys up to its last row, base / 32 + (w0 + WAVES (k + 1)) / G half tiles, with w0 the first wave that has new tokens.  A block costs
// those and OVER half tiles besides (its start and its output); all costs are in units of a G-th of half a tile.
//
// The blocks of all requests in a row are one axis of work of length T, which W workgroups per KV head cut into equal pieces: a
// piece starts and ends anywhere in a block, at a tile, and the states of a block that was cut are joined by a second kernel.  A
// single long request (the chunk no longer than what precedes it) takes whole blocks in step, so that the workgroups of an XCD read the same tiles
// at the same time, and only what is left over by them is cut.
// Every workgroup finds its pieces from the lengths by itself, and leaves where the first one starts for the joining kernel.
#pragma once
#include "paged.h"

namespace seka {

// Waves of a workgroup; half tiles that a block costs beside its keys; half tiles of a workgroup, at least (log2); no piece of fewer tiles;
// whether a block of which no more than half the waves have tokens costs half (the other waves share its keys); whether the lanes keep
// the lengths of up to 64 requests (five registers) or a piece reads them again.
template <int WAVES_, int OVER_, int LEAST_LOG2_, int SNAP_, bool HALVES_, bool HOLD_>
struct PipeShape {
  static constexpr bool HALVES = HALVES_, HOLD = HOLD_;
  static constexpr int WAVES = WAVES_, ROWS = 32 * WAVES_, OVER = OVER_, LEAST_LOG2 = LEAST_LOG2_, SNAP = SNAP_;
};
// bf16: stamps of the dense kernel say 4.7 tiles.  us, 32 / 8 heads, pieces of 6 tiles and 32 halves at least / of 2 and 8: one chunk of 512 over 512
// 39.0 / 28.1, 128 over 2048 42.1 / 34.1, four of up to 64 over 4096 43.4 / 32.8, 512 over 4096 57.4 / 53.5.
using PipeBf16 = PipeShape<8, 10, 3, 2, false, true>;
using PipeF32 = PipeShape<4, 2, 1, 1, true, false>;

// position of row 0; the first wave that has new tokens, of those that start there
__device__ __forceinline__ int pipe_first_row(const ChunkExtent& e) { return max(e.len - e.n, 0) & ~31; }
__device__ __forceinline__ int pipe_first_wave(const ChunkExtent& e, int G) { return (unsigned)((max(e.len - e.n, 0) & 31) * G) / 32u; }

struct PipeCut {
  int b, k, t;           // request, block, tile
};

template <class SHAPE>
struct PipePlan {
  static constexpr int WAVES = SHAPE::WAVES;
  ChunkRows r;
  PagedCache c;
  ChunkExtent mine;      // request `lane`, where there are no more than 64
  long long ends;        // and the half tiles of the requests up to it
  long long T, per;      // cost of all blocks; of a workgroup
  int G, W;              // workgroups that get work
  int rem, rounds;       // a single long request: blocks that are cut, whole blocks per workgroup; rounds = 0: everything is cut

  __device__ __forceinline__ PipePlan(const ChunkRows& rows, const PagedCache& cache, int width, int group) : r(rows), c(cache), mine{0, 0, 0}, ends(0), G(group) {
    T = 0;
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < r.B; b0 += 64) {
      ChunkExtent e = {0, 0, 0};
      if (b0 + lane < r.B) e = chunk_extent(r, c, b0 + lane);
      mine = e;
      ends = sums(work(e));
      T += uniform(__shfl(ends, 63));
    }
    const long long fill = T < 0x80000000ll ? ((uint32_t)T >> SHAPE::LEAST_LOG2) / (uint32_t)G : (T >> SHAPE::LEAST_LOG2) / G;
    W = (int)(fill < 1 ? 1 : fill < width ? fill : width);
    per = T < 0x80000000ll ? (long long)(((uint32_t)T + (uint32_t)W - 1) / (uint32_t)W) : (T + W - 1) / W;
    rem = rounds = 0;
    if (r.B == 1) {
      const ChunkExtent e = extent(0);
      const int nb = blocks(e);
      if (nb >= W && pipe_first_row(e) >= e.n) {
        rounds = nb / W;
        rem = nb - rounds * W;
        // the whole blocks count in full in cut(), so here too: their sums then rise and fall once from workgroup to workgroup, and the cuts never go back
        per = (before(e, nb) + W - 1) / W;
      }
    }
  }

  __device__ __forceinline__ static int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
  __device__ __forceinline__ static long long uniform(long long v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)((unsigned long long)v >> 32));
    return (long long)((unsigned long long)hi << 32 | lo);
  }
  __device__ __forceinline__ static long long sums(long long v) {      // inclusive, over the wave's lanes
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long o = __shfl_up(v, d);
      if (lane >= d) v += o;
    }
    return v;
  }
  __device__ __forceinline__ ChunkExtent extent(int b) const {
    ChunkExtent e;
    if (SHAPE::HOLD && r.B <= 64) {
      e.row0 = __builtin_amdgcn_readlane(mine.row0, b);
      e.n = __builtin_amdgcn_readlane(mine.n, b);
      e.len = __builtin_amdgcn_readlane(mine.len, b);
    } else {
      e = chunk_extent(r, c, b);
      e.row0 = uniform(e.row0);
      e.n = uniform(e.n);
      e.len = uniform(e.len);
    }
    return e;
  }
  __device__ __forceinline__ int blocks(const ChunkExtent& e) const {
    if (e.n <= 0 || e.len <= 0) return 0;
    return (waves(e) + WAVES - 1) / WAVES;
  }
  __device__ __forceinline__ int waves(const ChunkExtent& e) const { return (int)((unsigned)((e.len - pipe_first_row(e)) * G + 31) / 32u) - pipe_first_wave(e, G); }
  __device__ __forceinline__ bool half(const ChunkExtent& e, int k) const { return SHAPE::HALVES && waves(e) - WAVES * k <= WAVES / 2; }
  __device__ __forceinline__ int tiles(const ChunkExtent& e, int k) const {
    const int rows = 32 * (pipe_first_wave(e, G) + WAVES * (k + 1));        // behind first_row, up to the block's end
    return (min(e.len, pipe_first_row(e) + (int)((unsigned)(rows - 1) / (unsigned)G) + 1) - 1) / 64 + 1;
  }
  // cost of the blocks 0 .. k - 1
  __device__ __forceinline__ long long of_each(const ChunkExtent& e) const { return (long long)(pipe_first_row(e) / 32 + SHAPE::OVER) * G + pipe_first_wave(e, G); }
  __device__ __forceinline__ long long before(const ChunkExtent& e, long long k) const { return k * of_each(e) + WAVES * (k * (k + 1) / 2); }
  __device__ __forceinline__ long long work(const ChunkExtent& e) const {
    const int nb = blocks(e);
    const long long all = before(e, nb);
    return nb > 0 && half(e, nb - 1) ? (all + before(e, nb - 1)) / 2 : all;
  }

  // block k's index of round i for workgroup w: back and forth
  __device__ __forceinline__ int whole(int w, int i) const { return rem + i * W + (i & 1 ? W - 1 - w : w); }

  // Where workgroup w's piece of the axis starts (w = W: where the axis ends).
  __device__ __forceinline__ PipeCut cut(int w) const {
    long long x = per * w;
    if (rounds > 0) {
      // the whole blocks of the workgroups before w are theirs already
      const ChunkExtent e = extent(0);
      long long theirs = 0;
      for (int i = 0; i < rounds; ++i) {
        const long long first = rem + (long long)i * W + (i & 1 ? W - w : 0);      // w blocks from here
        theirs += before(e, first + w) - before(e, first);
      }
      const long long all = before(e, rem);
      x = w == W ? all : x - theirs;
      x = x < 0 ? 0 : x > all ? all : x;
      return at(e, 0, rem, x);
    }
    if (x >= T) return PipeCut{r.B, 0, 0};
    const int lane = threadIdx.x & 63;
    long long passed = 0;
    for (int b0 = 0; b0 < r.B; b0 += 64) {
      const bool held = SHAPE::HOLD && r.B <= 64;
      ChunkExtent e = mine;
      if (!held) {
        e = ChunkExtent{0, 0, 0};
        if (b0 + lane < r.B) e = chunk_extent(r, c, b0 + lane);
      }
      const long long own = work(e), upto = held ? ends : sums(own);
      const unsigned long long hit = __ballot(x - passed < upto);
      if (hit != 0ull) {
        const int l = __builtin_ctzll(hit);
        const long long start = passed + uniform(__shfl(upto - own, l));
        const ChunkExtent eb = extent(b0 + l);
        return at(eb, b0 + l, blocks(eb), x - start);
      }
      passed += uniform(__shfl(upto, 63));
    }
    return PipeCut{r.B, 0, 0};
  }

  // The place x into the first nb blocks of a request.
  __device__ __forceinline__ PipeCut at(const ChunkExtent& e, int b, int nb, long long x) const {
    constexpr float s = WAVES;
    // the last block that starts at x or before: s k (k + 1) / 2 + k f = x, put right by whole blocks (fp32: off by a few of millions)
    const float f = (float)of_each(e) + 0.5f * s;
    const float root = 2.f * (float)x / (f + sqrtf(f * f + 2.f * s * (float)x));
    int k = min(max((int)root, 0), nb);
    while (k > 0 && before(e, k) > x) --k;
    while (k < nb && before(e, k + 1) <= x) ++k;
    k = uniform(k);
    if (k >= nb) return PipeCut{b, nb, 0};
    const long long into = ((x - before(e, k)) << (half(e, k) ? 1 : 0)) - (long long)SHAPE::OVER * G;      // less than of_each and WAVES k
    const int n = tiles(e, k), t = uniform((int)(into < 0 ? 0u : (uint32_t)into / (uint32_t)(2 * G)));
    if (t < SHAPE::SNAP) return PipeCut{b, k, 0};
    if (n - t < SHAPE::SNAP) return PipeCut{b, k + 1, 0};
    return PipeCut{b, k, t};
  }
};

// What a workgroup does next: tiles t0 .. t1 - 1 of block k of request b, of n.
struct PipePiece {
  int b, k, t0, t1, n;
  ChunkExtent e;
  bool whole;            // nothing to join
};

// The pieces of workgroup w in turn.
template <class SHAPE>
struct PipePieces {
  PipePlan<SHAPE> p;
  int w, round;
  PipeCut now, end, start;

  __device__ __forceinline__ PipePieces(const ChunkRows& rows, const PagedCache& cache, int width, int group, int workgroup)
      : p(rows, cache, width, group), w(workgroup), round(0) {
    now = end = start = PipeCut{p.r.B, 0, 0};
    if (w >= p.W) {
      round = p.rounds;
      return;
    }
    start = now = p.cut(w);
    end = p.cut(w + 1);
  }
  __device__ __forceinline__ bool next(PipePiece& out) {
    while (now.b < p.r.B && (now.b < end.b || (now.b == end.b && (now.k < end.k || (now.k == end.k && now.t < end.t))))) {
      const ChunkExtent e = p.extent(now.b);
      if (now.k >= p.blocks(e)) {
        now = PipeCut{now.b + 1, 0, 0};
        continue;
      }
      const int n = p.tiles(e, now.k);
      const bool last = now.b == end.b && now.k == end.k;
      out = PipePiece{now.b, now.k, now.t, last ? end.t : n, n, e, false};
      out.whole = out.t0 == 0 && out.t1 == n;
      now = last ? end : PipeCut{now.b, now.k + 1, 0};
      if (out.t1 > out.t0) return true;
    }
    if (round < p.rounds) {
      const ChunkExtent e = p.extent(0);
      const int k = p.whole(w, round), n = p.tiles(e, k);
      ++round;
      out = PipePiece{0, k, 0, n, n, e, true};
      return true;
    }
    return false;
  }
  // a start inside a block that is the next workgroup's too: no tile, and no state
  __device__ __forceinline__ int4 note() const {
    const bool none = start.t > 0 && start.b == end.b && start.k == end.k && start.t == end.t;
    return make_int4(start.b, start.k, start.t, none);
  }
  // where the state of a piece that is not whole lies: each workgroup has at most two of them
  __device__ __forceinline__ int slot(const PipePiece& x) const { return 2 * w + (x.t0 > 0 ? 0 : 1); }
};

// New tokens that see no key (more of them than cached tokens): the requests item, item + width, .. of a KV head.
template <typename T, int D>
__device__ __forceinline__ void pipe_rows_without_keys(const ChunkArgs& pg, int item, int h) {
  const int lane = threadIdx.x & 63, G = pg.Hq / pg.Hkv;
  constexpr int PIECES = D * (int)sizeof(T) / 16;
  for (int b0 = 0; b0 < pg.r.B; b0 += 64) {
    ChunkExtent e = {0, 0, 0};
    const int mine = b0 + lane;
    if (mine < pg.r.B && mine % pg.width == item) e = chunk_extent(pg.r, pg.c, mine);
    unsigned long long todo = __ballot(e.n > e.len);
    for (; todo; todo &= todo - 1) {       // rare: lengths that do not count the new tokens
      const int l = __builtin_ctzll(todo);
      const int rows = __shfl(e.n - e.len, l), row0 = __shfl(e.row0, l);
      for (int x = threadIdx.x; x < rows * G * PIECES; x += blockDim.x) {
        const size_t row = (size_t)(row0 + x / (G * PIECES)) * pg.Hq + h * G;
        reinterpret_cast<uint4*>(static_cast<T*>(pg.O) + row * D)[x % (G * PIECES)] = make_uint4(0, 0, 0, 0);
      }
      if (pg.lse)
        for (int x = threadIdx.x; x < rows * G; x += blockDim.x) pg.lse[(size_t)(h * G + x % G) * pg.r.total + row0 + x / G] = -INFINITY;
    }
  }
}

}  // namespace seka
