// Long chunks over a cache of pages, head dimension 128.
#include "chunk_pipe.h"
namespace seka {
hipError_t launch_chunk_pipe_d128(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) { return launch_chunk_pipe<128>(a, p, s); }
}  // namespace seka
