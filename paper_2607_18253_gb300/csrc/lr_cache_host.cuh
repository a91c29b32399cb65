// The handle of the paged-cache calls and the checks that they share (lr_cache_api.cu, lr_cache_tokens.cu).
#pragma once

#include <cmath>
#include <string>

#include "latency_router.h"
#include "lr_cache.cuh"

struct lr_cache {
    int device = 0;
    int sms = 0;
    lr_cache_config cfg{};
    lr::CacheDev dev{};
    bool bf16 = true;
    lr::CacheMaps maps{};
    struct Parts {  // workspace of an attention kernel
        float *o = nullptr;
        float2 *ml = nullptr;
        uint32_t *done = nullptr;
    } step, chunk, weigh;
    std::string err;
};

namespace lr {

inline int fail(lr_cache *c, int code, const char *msg) {
    try {
        c->err = msg;
    } catch (...) {
    }
    return code;
}

inline int cuda_fail(lr_cache *c, cudaError_t e, const char *what) {
    try {
        c->err = std::string(what) + ": " + cudaGetErrorString(e);
    } catch (...) {
    }
    return LR_ECUDA;
}

inline bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Strides (elements of `size` bytes) that keep every vector 16-byte aligned.
inline bool good_stride(int64_t s, int size) { return s >= 0 && s < (1ll << 56) && s * size % 16 == 0; }

// The checks that the calls share; 0 if the batch may be launched.  (rows: the call uses q_start)
inline const char *bad_batch(const lr_cache_batch *b, int32_t T, bool rows = true) {
    if (!b) return "null batch";
    if (T < 0) return "T < 0";
    if (b->num_seqs < 0) return "num_seqs < 0";
    if (b->num_seqs > 0 && ((rows && !b->q_start) || !b->kv_len || !b->block_table)) return "null batch array";
    if (b->max_q < 1) return "max_q < 1";
    if (b->max_blocks < 0 || b->table_stride < b->max_blocks) return "table_stride below max_blocks";
    return nullptr;
}

inline BatchDev batch_dev(const lr_cache_batch *b, int32_t T) {
    return BatchDev{b->num_seqs, b->max_q, T, b->max_blocks, b->q_start, b->kv_len, b->block_table, b->table_stride};
}

}  // namespace lr
