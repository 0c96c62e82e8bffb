// seka_attention_chunk for long chunks: the kernel that joins the blocks of rows that were cut (chunk_plan.h).
#pragma once
#include "chunk_plan.h"

namespace seka {

// blockIdx: x: workgroup w whose piece starts inside a block, y: KV head and some of its rows, four columns to a thread.  The block's
// states: the end of the piece before w, then the starts of w's and of every later piece that starts in it too.
constexpr int kJoinThreads = 256;
template <typename T, class SHAPE, int D>
__global__ __launch_bounds__(kJoinThreads) void chunk_pipe_join_kernel(ChunkArgs pg) {
  constexpr int ROWS = kJoinThreads / (D / 4), PARTS = SHAPE::ROWS / ROWS;
  const int w = blockIdx.x + 1, h = blockIdx.y / PARTS, part = blockIdx.y % PARTS, G = pg.Hq / pg.Hkv;
  const int lane = threadIdx.x & 63;
  const int4 here = pg.cuts[w], prev = pg.cuts[w - 1];
  int4 mine = pg.cuts[min(w + lane, pg.width - 1)];
  if (here.z == 0 || here.x >= pg.r.B) return;
  if (prev.x == here.x && prev.y == here.y && prev.z > 0) return;      // an earlier workgroup's
  int pieces = 1;
  for (int v = w;; mine = pg.cuts[min(v + lane, pg.width - 1)]) {      // this one and those behind it that start in the same block
    const unsigned long long other = ~__ballot(v + lane < pg.width && mine.x == here.x && mine.y == here.y && mine.z > 0);
    pieces += other ? __builtin_ctzll(other) : 64;
    v += 64;
    if (other || v >= pg.width) break;
  }
  const ChunkExtent e = chunk_extent(pg.r, pg.c, here.x);
  const int r = part * ROWS + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4;      // row of the workgroup
  const int ctx = e.len - e.n, base = pipe_first_row(e);
  const unsigned row = 32u * pipe_first_wave(e, G) + here.y * SHAPE::ROWS + r, at = row / (unsigned)G;
  const int hq = h * G + (int)(row - at * G), pos = base + (int)at, i = pos - ctx;
  if (pos < max(ctx, 0) || i >= e.n) return;
  const size_t stride = (size_t)2 * pg.Hkv * SHAPE::ROWS * (D + 4);      // from a slot of one workgroup to the next one's
  const float* first = pg.part + ((size_t)(2 * w) * pg.Hkv + h) * SHAPE::ROWS * (D + 4) + (size_t)r * (D + 4);       // slot 2 w; the end before it: 2 w - 1
  const float* before = first - stride / 2;
  // (loads of the two states of a block cut once are on their way together)
  const float mb = before[D], lb = before[D + 1];
  const f32x4 ob = *reinterpret_cast<const f32x4*>(before + d);
  float m1 = first[D], l1 = first[D + 1];
  f32x4 o1 = *reinterpret_cast<const f32x4*>(first + d);
  if (here.w) {                            // a piece of no tile has left nothing there
    m1 = mb;
    l1 = 0.f;
    o1 = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float m = fmaxf(mb, m1);
#pragma unroll 4
  for (int s = 1; s < pieces - 1; ++s)
    if (!pg.cuts[w + s].w) m = fmaxf(m, first[s * stride + D]);
  const float f0 = __builtin_amdgcn_exp2f(mb - m), f1 = __builtin_amdgcn_exp2f(m1 - m);
  float l = lb * f0 + l1 * f1;
  f32x4 o = ob * f0 + o1 * f1;
#pragma unroll 4
  for (int s = 1; s < pieces - 1; ++s) {
    if (pg.cuts[w + s].w) continue;
    const float* ps = first + s * stride;
    const float f = __builtin_amdgcn_exp2f(ps[D] - m);
    l += ps[D + 1] * f;
    o += *reinterpret_cast<const f32x4*>(ps + d) * f;
  }
  const float inv = 1.f / l;
  T* O = static_cast<T*>(pg.O) + ((size_t)(e.row0 + i) * pg.Hq + hq) * D + d;
  if constexpr (sizeof(T) == 2) {
    bf16x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (__bf16)(o[k] * inv);
    *reinterpret_cast<bf16x4*>(O) = v;
  } else {
    *reinterpret_cast<f32x4*>(O) = o * inv;
  }
  if (pg.lse && d == 0) pg.lse[(size_t)hq * pg.r.total + e.row0 + i] = m * 0.6931471805599453f + logf(l);
}

struct PipeChunkPlan {
  int width;             // workgroups per KV head
  size_t smem, cuts, workspace;          // cuts: their offset in the workspace
};
hipError_t launch_chunk_block_f32(const ChunkArgs& a, int D, const PipeChunkPlan& p, hipStream_t s);

template <typename T, class SHAPE, int D>
void launch_chunk_join(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) {
  if (p.width > 1)
    hipLaunchKernelGGL((chunk_pipe_join_kernel<T, SHAPE, D>), dim3(p.width - 1, a.Hkv * SHAPE::ROWS / (kJoinThreads / (D / 4))), dim3(kJoinThreads), 0, s, a);
}

}  // namespace seka
