// Attention of few rows over a paged KV cache: the kernels of causal batches, and the calls of all (lr_attend_step.cuh).
#include "lr_attend_step.cuh"

namespace lr {

int attend_step_ctas(int sms) { return 4 * sms; }

cudaError_t attend_step_init() {
    const cudaError_t e = step_init<false>();
    return e == cudaSuccess ? tree_step_init() : e;
}

cudaError_t launch_attend_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st) {
    return a.tree ? launch_tree_step(a, bf16, fmt, rows, sms, st) : launch_step<false>(a, bf16, fmt, rows, sms, st);
}

}  // namespace lr
