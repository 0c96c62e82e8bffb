// How the blocks of query rows of a batch over a cache of pages are dealt to workgroups (attention_chunk_pipe_kernel).
//
// A request's new tokens are its last n of len cached ones.  Its rows are cut into blocks of BQ at positions that are multiples of
// 32, so that a wave's 32 rows end at half a key tile; the block that starts at base + k BQ sees the keys up to its last row, which
// is base / 32 + (k + 1) BQ / 32 half tiles.  A block costs those and kOver half tiles besides (its start and its output).
//
// The blocks of all requests in a row are one axis of work of length T, which W workgroups per head chunk cut into equal pieces: a
// piece starts and ends anywhere in a block, at a tile, and the states of a block that was cut are joined by a second kernel.  A
// single long request (the chunk no longer than what precedes it) takes whole blocks in step, so that the workgroups of an XCD read the same tiles
// at the same time, and only what is left over by them is cut.
// Every workgroup finds its pieces from the lengths by itself, and leaves where the first one starts for the joining kernel.
#pragma once
#include "paged.h"

namespace seka {

constexpr int kPipeOver = 10;            // half tiles that a block costs beside its keys (stamps of the dense kernel: 4.7 tiles)
// No piece of fewer tiles; half tiles of a workgroup, at least (log2).  us, 32 / 8 heads, 6 tiles and 32 halves / 2 and 8: one chunk of 512 over 512
// 39.0 / 28.1, 128 over 2048 42.1 / 34.1, four of up to 64 over 4096 43.4 / 32.8, 512 over 4096 57.4 / 53.5.
constexpr int kPipeSnap = 2;
constexpr int kPipeLeastLog2 = 3;

struct PipeCut {
  int b, k, t;           // request, block, tile
};

template <int BQ>
struct PipePlan {
  static constexpr long long s = BQ / 32;
  ChunkRows r;
  PagedCache c;
  ChunkExtent mine;      // request `lane`, where there are no more than 64
  long long ends;        // and the half tiles of the requests up to it
  long long T, per;      // half tiles of all blocks; of a workgroup
  int W;                 // workgroups that get work
  int rem, rounds;       // a single long request: blocks that are cut, whole blocks per workgroup; rounds = 0: everything is cut

  __device__ __forceinline__ PipePlan(const ChunkRows& rows, const PagedCache& cache, int width) : r(rows), c(cache), mine{0, 0, 0}, ends(0) {
    T = 0;
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < r.B; b0 += 64) {
      ChunkExtent e = {0, 0, 0};
      if (b0 + lane < r.B) e = chunk_extent(r, c, b0 + lane);
      mine = e;
      ends = sums(work(e));
      T += uniform(__shfl(ends, 63));
    }
    const long long fill = T >> kPipeLeastLog2;
    W = (int)(fill < 1 ? 1 : fill < width ? fill : width);
    per = T < 0x80000000ll ? (long long)(((uint32_t)T + (uint32_t)W - 1) / (uint32_t)W) : (T + W - 1) / W;
    rem = rounds = 0;
    if (r.B == 1) {
      const ChunkExtent e = extent(0);
      const int nb = blocks(e);
      if (nb >= W && (long long)first_row(e) >= (long long)nb * BQ) {
        rounds = nb / W;
        rem = nb - rounds * W;
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
    if (r.B <= 64) {
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
  // position of the first block's first row
  __device__ __forceinline__ static int first_row(const ChunkExtent& e) { return max(e.len - e.n, 0) & ~31; }
  __device__ __forceinline__ static int blocks(const ChunkExtent& e) { return e.n > 0 && e.len > 0 ? (e.len - first_row(e) + BQ - 1) / BQ : 0; }
  __device__ __forceinline__ static int tiles(const ChunkExtent& e, int k) { return (min(e.len, first_row(e) + (k + 1) * BQ) - 1) / 64 + 1; }
  // half tiles of the blocks 0 .. k - 1
  __device__ __forceinline__ static long long before(const ChunkExtent& e, long long k) {
    return k * (first_row(e) / 32 + kPipeOver) + s * (k * (k + 1) / 2);
  }
  __device__ __forceinline__ static long long work(const ChunkExtent& e) { return before(e, blocks(e)); }

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
      const bool held = r.B <= 64;
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

  // The place x half tiles into the first nb blocks of a request.
  __device__ __forceinline__ static PipeCut at(const ChunkExtent& e, int b, int nb, long long x) {
    // the last block that starts at x or before: s k (k + 1) / 2 + k f = x, put right by whole blocks (fp32: off by a few of millions)
    const float f = (float)(first_row(e) / 32 + kPipeOver) + 0.5f * s;
    const float root = 2.f * (float)x / (f + sqrtf(f * f + 2.f * s * (float)x));
    int k = min(max((int)root, 0), nb);
    while (k > 0 && before(e, k) > x) --k;
    while (k < nb && before(e, k + 1) <= x) ++k;
    k = uniform(k);
    if (k >= nb) return PipeCut{b, nb, 0};
    const long long into = x - before(e, k) - kPipeOver;
    const int n = tiles(e, k), t = uniform((int)(into < 0 ? 0 : into / 2));
    if (t < kPipeSnap) return PipeCut{b, k, 0};
    if (n - t < kPipeSnap) return PipeCut{b, k + 1, 0};
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
template <int BQ>
struct PipePieces {
  PipePlan<BQ> p;
  int w, round;
  PipeCut now, end, start;

  __device__ __forceinline__ PipePieces(const ChunkRows& rows, const PagedCache& cache, int width, int workgroup)
      : p(rows, cache, width), w(workgroup), round(0) {
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
      if (now.k >= PipePlan<BQ>::blocks(e)) {
        now = PipeCut{now.b + 1, 0, 0};
        continue;
      }
      const int n = PipePlan<BQ>::tiles(e, now.k);
      const bool last = now.b == end.b && now.k == end.k;
      out = PipePiece{now.b, now.k, now.t, last ? end.t : n, n, e, false};
      out.whole = out.t0 == 0 && out.t1 == n;
      now = last ? end : PipeCut{now.b, now.k + 1, 0};
      if (out.t1 > out.t0) return true;
    }
    if (round < p.rounds) {
      const ChunkExtent e = p.extent(0);
      const int k = p.whole(w, round), n = PipePlan<BQ>::tiles(e, k);
      ++round;
      out = PipePiece{0, k, 0, n, n, e, true};
      return true;
    }
    return false;
  }
  // where the state of a piece that is not whole lies: each workgroup has at most two of them
  __device__ __forceinline__ int slot(const PipePiece& x) const { return 2 * w + (x.t0 > 0 ? 0 : 1); }
};

}  // namespace seka
