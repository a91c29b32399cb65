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
    const uint32_t *tree;        // drafted tokens that each new token sees, a bit each; null: causal
    int64_t tree_t;              // words from a token's to the next one's
    int32_t row_lo, row_hi;      // sequences with this many rows (tokens x query heads a KV head) are this launch's
    float *part_o;               // [slots][rows][DP] sums of weighted V
    float2 *part_ml;             // [slots][rows] running maximum (log2) and sum
    uint32_t *done;              // parts finished of the unit that began in a CTA ([CTAs]; chunk kernel [3][CTAs][8 warps]); zero
                                 // between calls
};
constexpr int kStepRows = 16;   // rows of a unit of the step kernel, at most
constexpr int kTreeRows = 128;  // rows of a tree that are the step kernel's, in tiles of 16, at most; of 32 tokens, a word of their masks
constexpr int kTreeLittle = 400000;  // tokens x KV heads x tiles of 16 rows that are little
cudaError_t launch_attend_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st);
cudaError_t attend_step_init();
int attend_step_ctas(int sms);  // CTAs of a launch, at most
constexpr int kChunkCounts = 24;  // counters of finished parts a CTA
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
// The map of a launch's queries: boxes of 64 elements of as many tokens' rows of a KV head as 128 holds; false if there can be none.
bool encode_rows(const AttendLaunch &a, bool bf16, CUtensorMap &map);
// The kernels of trees (a.tree), which the above launch.
cudaError_t tree_step_init();
cudaError_t launch_tree_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st);
cudaError_t tree_chunk_init();
cudaError_t launch_tree_chunk(const AttendLaunch &a, const CacheMaps &m, bool bf16, int fmt, int ctas, cudaStream_t st);


// The weights that tokens have received (lr_weigh.cu): the batch and queries as for attention, lse as an input.
struct WeighLaunch {
    AttendLaunch a;
    float *w;
    int64_t wb, wt, wh;  // strides of block, token, head in floats
    float decay;
    float lse_log2, lse_log2_rest;  // scale_log2 / scale: with the rounding of scale_log2 in it, so that it cancels where a score is near its lse
};
cudaError_t launch_weigh(const WeighLaunch &a, const CacheMaps &m, bool bf16, int fmt, int sms, cudaStream_t st);
// (its kernels: of sequences of `rows` rows at most, 8 or 16; of others, one CTA an SM, whose parts of 256 tokens are joined)
cudaError_t launch_weigh_step(const WeighLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st);
cudaError_t launch_weigh_chunk(const WeighLaunch &a, const CacheMaps &m, bool bf16, int fmt, int sms, cudaStream_t st);
cudaError_t weigh_init();

// The tokens that a cache keeps (lr_select.cu).
struct SelectLaunch {
    CacheDev c;
    BatchDev b;
    const float *w;
    int64_t wb, wt, wh;
    const int32_t *budget;  // or null: cap
    int32_t cap, sinks, recent;
    int32_t *kept, *count;
    int32_t cluster, hold;  // (set by the launch) CTAs a list, keys that a CTA holds
};
cudaError_t launch_select(const SelectLaunch &a, int sms, cudaStream_t st);
cudaError_t select_init();

// Tokens moved together, in place (lr_keep.cu).
struct KeepLaunch {
    CacheDev c;
    BatchDev b;
    const int32_t *kept;     // [n][heads][cap]
    int64_t kept_s, kept_h;  // strides of sequence and head; kept_h 0: one list for all heads
    const int32_t *count, *start;
    int32_t cap;
    float *w;                // or null
    int64_t wb, wt, wh;
    int32_t vector, pieces, cluster;  // (set by the launch) bytes of a vector, parts that it is moved in, CTAs a list of such parts
};
cudaError_t keep_init();
cudaError_t launch_keep(const KeepLaunch &a, int fmt, int sms, cudaStream_t st);

// As launch_chained, in clusters of `cluster` CTAs.
template <typename A>
cudaError_t launch_clusters(void (*k)(const A), unsigned grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t st, const A &a) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k, A(a));
}

}  // namespace lr
