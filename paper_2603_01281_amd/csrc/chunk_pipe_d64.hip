// Long chunks over a cache of pages, head dimension 64.
#include "chunk_pipe.h"
namespace seka {
hipError_t launch_chunk_pipe_d64(const ChunkArgs& a, const PipeChunkPlan& p, hipStream_t s) { return launch_chunk_pipe<64>(a, p, s); }
}  // namespace seka
