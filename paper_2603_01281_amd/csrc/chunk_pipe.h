// seka_attention_chunk for long chunks, bf16: the software-pipelined prefill kernel over pages (attn_bf16_pipe_kernel.h).
// One workgroup of eight waves to a compute unit; tiles of 64 keys and values go from the pages straight into LDS, their page numbers a tile ahead.
// MFMA-bound under the chip's power limit: 2048 new tokens over 31111, 32 / 8 heads, D = 128, 820 us, 1.23 PFLOP/s (the kernel without pages
// reaches 1.25); nine requests of up to 700 over 6001, 28 / 4 heads, 150 us, 0.9 PFLOP/s: the cuts' states (up to 68 MB written and read) and
// the rows of blocks that no token fills.  The probabilities' sums are those before their rounding, on the vector unit, so that lse is good to fp32.
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
