// Attention of many rows over a paged KV cache: the kernels of trees of drafted tokens (lr_attend_chunk.cuh).
#include "lr_attend_chunk.cuh"

namespace lr {

cudaError_t tree_chunk_init() { return chunk_init<true>(); }
cudaError_t launch_tree_chunk(const AttendLaunch &a, const CacheMaps &m, bool bf16, int fmt, int ctas, cudaStream_t st) {
    return launch_chunk<true>(a, m, bf16, fmt, ctas, st);
}

}  // namespace lr
