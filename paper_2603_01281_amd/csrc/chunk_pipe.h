// seka_attention_chunk for long chunks, bf16: the software-pipelined prefill kernel over pages (attn_bf16_pipe_kernel.h).
#pragma once
#include <algorithm>

#include "attn_bf16_pipe_kernel.h"
#include "chunk_join.h"

namespace seka {

template <int D>
__global__ __launch_bounds__(64 * PipeBf16::WAVES) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 2 : 8))) void chunk_pipe_kernel(ChunkArgs pg) {
  AttnArgs a = {};
  a.Q = pg.Q; a.K = pg.c.K; a.V = pg.c.V; a.O = pg.O; a.lse = pg.lse;
  a.Hq = pg.Hq; a.Hkv = pg.Hkv; a.D = D; a.scale = pg.scale;
  attention_bf16_pipe_body<D, 1, PipeBf16::WAVES, false, 1>(a, SteerArgs{}, pg);
}

hipError_t launch_chunk_pipe_d128(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s);
hipError_t launch_chunk_pipe_d64(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s);

template <int D>
hipError_t launch_chunk_pipe(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) {
  auto kernel = chunk_pipe_kernel<D>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.width * a.Hkv)), dim3(64 * PipeBf16::WAVES), p.smem, s, a);
  launch_chunk_join<uint16_t, PipeBf16, D>(a, p, s);
  return hipGetLastError();
}

}  // namespace seka
