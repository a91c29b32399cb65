// Layout shared by the paged-cache calls: the host side (lr_cache_api.cu), the store and
// load kernels (lr_cache_rw.cu) and the attention kernels (lr_attend_*.cu).
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "lr_internal.cuh"

namespace lr {

enum : int { kFmt16 = 0, kFmtE4M3 = 1, kFmtInt8 = 2 };
constexpr int kMaxTokens = 1 << 30;  // largest kv_len

// n / d for 0 <= n < 2^31 by one multiplication: m = ceil(2^(31 + s) / d) with 2^s >= d is
// below 2^32, and n * (m * d - 2^(31+s)) < 2^31 * 2^s, so the quotient is exact.
struct FastDiv {
    uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f{d, 0, 0};
    while ((1ull << f.s) < d) ++f.s;
    f.m = (uint32_t)(((1ull << (31 + f.s)) + d - 1) / d);
    return f;
}
__device__ __forceinline__ int quot(int n, const FastDiv &f) {
    return (int)((unsigned long long)(uint32_t)n * f.m >> (31 + f.s));
}

struct CacheDev {
    char *k, *v;
    float *ks, *vs;
    int64_t sb, st, sh;     // strides of block, token, head in BYTES
    int64_t ssb, sst, ssh;  // strides of the scales in floats
    int32_t H, Hq, G, D;    // KV heads, query heads, query heads a KV head, head size
    int32_t nb, b;          // blocks, tokens a block
    FastDiv div_b, div_g;
    int32_t *status;
    const float *nan;  // one
};

struct BatchDev {
    int32_t n, max_q, T, max_blocks;
    const int32_t *q_start, *kv_len, *table;
    int64_t table_stride;
};

__device__ __forceinline__ void report(int32_t *status, int code) { atomicCAS(status, 0, code); }

// Byte offset of (block, place) of token p of sequence s, -1 if it has none.
__device__ __forceinline__ int64_t block_of(const CacheDev &c, const BatchDev &b, int s, int p, int &place) {
    const int i = quot(p, c.div_b);
    place = p - i * c.b;
    if (i >= b.max_blocks) return -1;
    const int blk = __ldg(b.table + (int64_t)s * b.table_stride + i);
    return (uint32_t)blk < (uint32_t)c.nb ? (int64_t)blk : -1;
}

// ---- launches ----
struct RwLaunch {
    CacheDev c;
    BatchDev b;
    const char *k_in, *v_in;
    int64_t in_t, in_h;  // bytes
    char *k_out, *v_out;
};
cudaError_t launch_cache_write(const RwLaunch &a, bool bf16, int fmt, cudaStream_t st);
cudaError_t launch_cache_read(const RwLaunch &a, bool bf16, int fmt, bool f32, cudaStream_t st);

// Partial results of the attention kernels: a unit (sequence, KV head, tile of rows) whose cached
// tokens are split over several CTAs is joined by the last of them to finish.  A CTA works
// through one contiguous range of the batch's tiles, so at most its first and its last
// unit are shared with others: two slots of `rows` rows each.
struct AttendLaunch {
    CacheDev c;
    BatchDev b;
    const char *q;
    char *out;
    float *lse;
    int64_t q_t, q_h, o_t, o_h;  // bytes
    float scale_log2;            // scale * log2(e)
    int32_t window, sinks;
    int32_t row_lo, row_hi;      // sequences with this many rows (tokens x query heads a KV head) are this launch's
    float *part_o;               // [slots][rows][DP] sums of weighted V
    float2 *part_ml;             // [slots][rows] running maximum (log2) and sum
    uint32_t *done;              // parts finished of the unit that began in a CTA ([CTAs]; chunk kernel [CTAs][8 warps]); zero
                                 // between calls
};
constexpr int kStepRows = 16;   // rows of a unit of the step kernel, at most
cudaError_t launch_attend_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st);
cudaError_t attend_step_init();
int attend_step_ctas(int sms);  // CTAs of a launch, at most
constexpr int kChunkRows = 256;  // rows of a unit of the chunk kernel; one CTA an SM
// Tensor maps of a 16-bit cache's K and V: boxes of 64 elements of `box` tokens, the largest number that
// divides a block and the chunk kernel's tiles; box 0: none (blocks that are no multiple of 8 tokens).
struct CacheMaps {
    CUtensorMap k, v;
    int32_t box;
};
int encode_maps(const CacheDev &c, bool bf16, CacheMaps &m);  // the box, 0 if there can be none
cudaError_t launch_attend_chunk(const AttendLaunch &a, const CacheMaps &m, bool bf16, int fmt, int ctas, cudaStream_t st);
cudaError_t attend_chunk_init();

}  // namespace lr
