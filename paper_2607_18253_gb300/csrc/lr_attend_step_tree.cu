// Attention of few rows over a paged KV cache: the kernels of trees of drafted tokens (lr_attend_step.cuh).
#include "lr_attend_step.cuh"

namespace lr {

cudaError_t tree_step_init() { return step_init<true>(); }
cudaError_t launch_tree_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st) {
    return launch_step<true>(a, bf16, fmt, rows, sms, st);
}

}  // namespace lr
