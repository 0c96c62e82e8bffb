// seka_attention_chunk for long chunks, bf16: the software-pipelined prefill kernel over pages (attn_bf16_pipe_kernel.h), and the kernel that
// joins the blocks of rows that were cut.
#pragma once
#include <algorithm>

#include "attn_bf16_pipe_kernel.h"

namespace seka {

template <int D, int HPW, int RBW>
__global__ __launch_bounds__(64 * HPW * RBW) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 2 : 8))) void chunk_pipe_kernel(ChunkArgs pg) {
  AttnArgs a = {};
  a.Q = pg.Q; a.K = pg.c.K; a.V = pg.c.V; a.O = pg.O; a.lse = pg.lse;
  a.Hq = pg.Hq; a.Hkv = pg.Hkv; a.D = D; a.scale = pg.scale;
  attention_bf16_pipe_body<D, HPW, RBW, false, 1>(a, SteerArgs{}, pg);
}

// blockIdx: x: workgroup w whose piece starts inside a block, y: head chunk and 32 of its rows.  The block's states: the end of the piece before
// w, then the starts of w's and of every later piece that starts in it too.
template <int D, int HPW, int RBW>
__global__ __launch_bounds__(256) void chunk_pipe_join_kernel(ChunkArgs pg) {
  constexpr int BQ = 32 * RBW, PARTS = HPW * RBW;
  const int w = blockIdx.x + 1, hc = blockIdx.y / PARTS, part = blockIdx.y % PARTS, nHC = pg.Hq / HPW;
  const PipePlan<BQ> plan(pg.r, pg.c, pg.width);
  if (w >= plan.W) return;
  const PipeCut here = plan.cut(w);
  if (here.t == 0 || here.b >= pg.r.B) return;
  const PipeCut prev = plan.cut(w - 1);
  if (prev.b == here.b && prev.k == here.k && prev.t > 0) return;      // an earlier workgroup's
  int pieces = 2;
  for (int v = w + 1; v < plan.W; ++v) {
    const PipeCut later = plan.cut(v);
    if (later.b != here.b || later.k != here.k || later.t == 0) break;
    ++pieces;
  }
  const ChunkExtent e = plan.extent(here.b);
  const int ctx = e.len - e.n, hq = hc * HPW + part / RBW;
  const int pos0 = PipePlan<BQ>::first_row(e) + here.k * BQ + 32 * (part % RBW);
  const size_t stride = (size_t)2 * nHC * (HPW * BQ) * (D + 4);        // from a slot of one workgroup to the next one's
  const float* base = pg.part + ((size_t)(2 * w) * nHC + hc) * (HPW * BQ) * (D + 4) + (size_t)part * 32 * (D + 4);
  for (int idx = threadIdx.x; idx < 32 * (D / 4); idx += 256) {
    const int r = idx / (D / 4), d = idx % (D / 4) * 4, i = pos0 + r - ctx;
    if (pos0 + r < max(ctx, 0) || i >= e.n) continue;
    const float* ps = base + (size_t)r * (D + 4) - stride / 2;         // slot 2 w - 1
    float m = -1e30f, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < pieces; ++s) {
      const float m2 = ps[D], l2 = ps[D + 1];
      const f32x4 o2 = *reinterpret_cast<const f32x4*>(ps + d);
      const float mm = fmaxf(m, m2), f1 = __builtin_amdgcn_exp2f(m - mm), f2 = __builtin_amdgcn_exp2f(m2 - mm);
      m = mm;
      l = l * f1 + l2 * f2;
      o = o * f1 + o2 * f2;
      ps += s == 0 ? stride / 2 : stride;
    }
    const float inv = 1.f / l;
    bf16x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (__bf16)(o[k] * inv);
    *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(pg.O) + ((size_t)(e.row0 + i) * pg.Hq + hq) * D + d) = v;
    if (pg.lse && d == 0) pg.lse[(size_t)hq * pg.r.total + e.row0 + i] = m * 0.6931471805599453f + logf(l);
  }
}

struct PipeChunkPlan {
  int hpw, rbw;          // heads and blocks of 32 rows of a workgroup
  int width;             // workgroups per head chunk
  size_t smem, workspace;
};

hipError_t launch_chunk_pipe_d128(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s);
hipError_t launch_chunk_pipe_d64(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s);

template <int D, int HPW, int RBW>
hipError_t launch_chunk_pipe_cfg(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) {
  auto kernel = chunk_pipe_kernel<D, HPW, RBW>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem);
  if (e != hipSuccess) return e;
  const int nHC = a.Hq / HPW;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.width * nHC)), dim3(64 * HPW * RBW), p.smem, s, a);
  if (p.width > 1) hipLaunchKernelGGL((chunk_pipe_join_kernel<D, HPW, RBW>), dim3(p.width - 1, nHC * HPW * RBW), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_chunk_pipe(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) {
  if (p.hpw == 4) return launch_chunk_pipe_cfg<D, 4, 2>(a, p, s);
  if (p.hpw == 7) return launch_chunk_pipe_cfg<D, 7, 1>(a, p, s);
  if (p.hpw == 2) return launch_chunk_pipe_cfg<D, 2, 4>(a, p, s);
  return launch_chunk_pipe_cfg<D, 1, 8>(a, p, s);
}

}  // namespace seka
