// Host side of the paged-cache calls declared in include/latency_router.h: validation,
// workspace, launch shapes and the status word.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
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
    } step, chunk;
    std::string err;
};

namespace {

int fail(lr_cache *c, int code, const char *msg) {
    try {
        c->err = msg;
    } catch (...) {
    }
    return code;
}

int cuda_fail(lr_cache *c, cudaError_t e, const char *what) {
    try {
        c->err = std::string(what) + ": " + cudaGetErrorString(e);
    } catch (...) {
    }
    return LR_ECUDA;
}

void free_all(lr_cache *c) {
    cudaFree(c->dev.status);
    for (lr_cache::Parts *p : {&c->step, &c->chunk}) {
        cudaFree(p->o);
        cudaFree(p->ml);
        cudaFree(p->done);
    }
}

// Two slots of partial rows a CTA, and counters at zero.
cudaError_t alloc_parts(lr_cache::Parts &p, size_t ctas, size_t rows, size_t counters) {
    cudaError_t e = cudaMalloc(&p.o, 2 * ctas * rows * 128 * sizeof(float));
    if (e == cudaSuccess) e = cudaMalloc(&p.ml, 2 * ctas * rows * sizeof(float2));
    if (e == cudaSuccess) e = cudaMalloc(&p.done, counters * sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMemset(p.done, 0, counters * sizeof(uint32_t));
    return e;
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Strides (elements of `size` bytes) that keep every vector 16-byte aligned.
bool good_stride(int64_t s, int size) { return s >= 0 && s < (1ll << 56) && s * size % 16 == 0; }

// The checks that the calls share; 0 if the batch may be launched.
const char *bad_batch(const lr_cache_batch *b, int32_t T) {
    if (!b) return "null batch";
    if (T < 0) return "T < 0";
    if (b->num_seqs < 0) return "num_seqs < 0";
    if (b->num_seqs > 0 && (!b->q_start || !b->kv_len || !b->block_table)) return "null batch array";
    if (b->max_q < 1) return "max_q < 1";
    if (b->max_blocks < 0 || b->table_stride < b->max_blocks) return "table_stride below max_blocks";
    return nullptr;
}

lr::BatchDev batch_dev(const lr_cache_batch *b, int32_t T) {
    return lr::BatchDev{b->num_seqs, b->max_q, T, b->max_blocks, b->q_start, b->kv_len, b->block_table, b->table_stride};
}

}  // namespace

extern "C" {

int lr_cache_create(const lr_cache_config *cfg, lr_cache **out) {
    if (!cfg || !out) return LR_EINVAL;
    *out = nullptr;
    lr_cache *c = new (std::nothrow) lr_cache();
    if (!c) return LR_ENOMEM;
    auto bail = [&](int code, const char *msg) {
        std::fprintf(stderr, "lr_cache_create: %s\n", msg);
        free_all(c);
        delete c;
        return code;
    };
    if (cfg->num_kv_heads < 1 || cfg->num_q_heads < cfg->num_kv_heads || cfg->num_q_heads > 1024 ||
        cfg->num_q_heads % cfg->num_kv_heads)
        return bail(LR_EINVAL, "num_q_heads must be a multiple of num_kv_heads, at most 1024");
    if (cfg->head_dim < 16 || cfg->head_dim > 128 || cfg->head_dim % 16)
        return bail(LR_EINVAL, "head_dim must be a multiple of 16 in [16, 128]");
    if (cfg->dtype != LR_BF16 && cfg->dtype != LR_FP16) return bail(LR_EINVAL, "dtype must be LR_BF16 or LR_FP16");
    if (cfg->format != LR_CACHE_16BIT && cfg->format != LR_CACHE_E4M3 && cfg->format != LR_CACHE_INT8)
        return bail(LR_EINVAL, "format");
    if (cfg->block_size < 1 || cfg->block_size > 4096) return bail(LR_EINVAL, "block_size must be in [1, 4096]");
    if (cfg->num_blocks < 1) return bail(LR_EINVAL, "num_blocks must be positive");
    if (cfg->max_seqs < 1 || cfg->max_seqs > (1 << 16)) return bail(LR_EINVAL, "max_seqs must be in [1, 65536]");
    if (!cfg->k || !cfg->v || !aligned16(cfg->k) || !aligned16(cfg->v))
        return bail(LR_EINVAL, "k and v must be 16-byte aligned device pointers");
    const int size = cfg->format == LR_CACHE_16BIT ? 2 : 1;
    if (!good_stride(cfg->block_stride, size) || !good_stride(cfg->token_stride, size) || !good_stride(cfg->head_stride, size))
        return bail(LR_EINVAL, "strides must be non-negative multiples of 16 bytes");
    if (cfg->format != LR_CACHE_16BIT &&
        (!cfg->k_scale || !cfg->v_scale || cfg->scale_block_stride < 0 || cfg->scale_token_stride < 0 || cfg->scale_head_stride < 0))
        return bail(LR_EINVAL, "8-bit formats need k_scale and v_scale with non-negative strides");
    c->cfg = *cfg;
    c->bf16 = cfg->dtype == LR_BF16;
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, c->device);
    if (e == cudaSuccess) e = lr::attend_step_init();
    if (e == cudaSuccess) e = lr::attend_chunk_init();
    if (e != cudaSuccess) return bail(LR_ECUDA, cudaGetErrorString(e));
    lr::CacheDev &d = c->dev;
    d.k = static_cast<char *>(cfg->k);
    d.v = static_cast<char *>(cfg->v);
    d.ks = cfg->k_scale;
    d.vs = cfg->v_scale;
    d.sb = cfg->block_stride * size;
    d.st = cfg->token_stride * size;
    d.sh = cfg->head_stride * size;
    d.ssb = cfg->scale_block_stride;
    d.sst = cfg->scale_token_stride;
    d.ssh = cfg->scale_head_stride;
    d.H = cfg->num_kv_heads;
    d.Hq = cfg->num_q_heads;
    d.G = d.Hq / d.H;
    d.D = cfg->head_dim;
    d.nb = cfg->num_blocks;
    d.b = cfg->block_size;
    d.div_b = lr::fast_div(d.b);
    d.div_g = lr::fast_div(d.G);
    if (cfg->format == LR_CACHE_16BIT) lr::encode_maps(d, c->bf16, c->maps);
    e = cudaMalloc(&d.status, 16);
    const uint32_t words[4] = {0, 0x7fffffffu, 0, 0};  // the status word, a NaN
    if (e == cudaSuccess) e = cudaMemcpy(d.status, words, sizeof(words), cudaMemcpyHostToDevice);
    d.nan = reinterpret_cast<const float *>(d.status + 1);
    if (e == cudaSuccess) e = alloc_parts(c->step, lr::attend_step_ctas(c->sms), lr::kStepRows, lr::attend_step_ctas(c->sms));
    if (e == cudaSuccess) e = alloc_parts(c->chunk, c->sms, lr::kChunkRows, 8 * (size_t)c->sms);
    if (e != cudaSuccess) return bail(LR_ENOMEM, cudaGetErrorString(e));
    // (what was set above, on the default stream, has to be there for streams that do not wait for it)
    e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return bail(LR_ECUDA, cudaGetErrorString(e));
    *out = c;
    return LR_OK;
}

int lr_cache_destroy(lr_cache *c) {
    if (!c) return LR_OK;
    cudaDeviceSynchronize();
    free_all(c);
    delete c;
    return LR_OK;
}

int lr_cache_write(lr_cache *c, const lr_cache_batch *b, int32_t T, const void *k, const void *v, int64_t token_stride,
                   int64_t head_stride, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, T)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (T == 0 || b->num_seqs == 0) return LR_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(c, LR_EINVAL, "k and v must be 16-byte aligned");
    if (!good_stride(token_stride, 2) || !good_stride(head_stride, 2))
        return fail(c, LR_EINVAL, "strides must be non-negative multiples of 16 bytes");
    lr::RwLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.c = c->dev;
    a.b = batch_dev(b, T);
    a.k_in = static_cast<const char *>(k);
    a.v_in = static_cast<const char *>(v);
    a.in_t = token_stride * 2;
    a.in_h = head_stride * 2;
    cudaError_t e = lr::launch_cache_write(a, c->bf16, c->cfg.format, (cudaStream_t)stream);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "cache write launch");
}

int lr_cache_read(lr_cache *c, const lr_cache_batch *b, int32_t T, int32_t out_dtype, void *k_out, void *v_out, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, T)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (out_dtype != c->cfg.dtype && out_dtype != LR_FP32) return fail(c, LR_EINVAL, "out_dtype must be the cache's dtype or LR_FP32");
    if (T == 0 || b->num_seqs == 0) return LR_OK;
    if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return fail(c, LR_EINVAL, "k_out and v_out must be 16-byte aligned");
    lr::RwLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.c = c->dev;
    a.b = batch_dev(b, T);
    a.k_out = static_cast<char *>(k_out);
    a.v_out = static_cast<char *>(v_out);
    cudaError_t e = lr::launch_cache_read(a, c->bf16, c->cfg.format, out_dtype == LR_FP32, (cudaStream_t)stream);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "cache read launch");
}

int lr_cache_attend(lr_cache *c, const lr_cache_batch *b, int32_t T, const void *q, int64_t q_token_stride,
                    int64_t q_head_stride, float scale, int32_t window, int32_t sinks, void *out, int64_t out_token_stride,
                    int64_t out_head_stride, float *lse_out, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, T)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (!(std::isfinite(scale) && scale > 0.0f)) return fail(c, LR_EINVAL, "scale must be finite and positive");
    if (window < 0 || window > lr::kMaxTokens || sinks < 0 || sinks > lr::kMaxTokens)
        return fail(c, LR_EINVAL, "window and sinks must be in [0, 2^30]");
    if (b->max_q > (1 << 20)) return fail(c, LR_EINVAL, "max_q must be at most 2^20");
    if (T == 0 || b->num_seqs == 0) return LR_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out)) return fail(c, LR_EINVAL, "q and out must be 16-byte aligned");
    if (!good_stride(q_token_stride, 2) || !good_stride(q_head_stride, 2) || !good_stride(out_token_stride, 2) ||
        !good_stride(out_head_stride, 2))
        return fail(c, LR_EINVAL, "strides must be non-negative multiples of 16 bytes");
    lr::AttendLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.c = c->dev;
    a.b = batch_dev(b, T);
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    a.lse = lse_out;
    a.q_t = q_token_stride * 2;
    a.q_h = q_head_stride * 2;
    a.o_t = out_token_stride * 2;
    a.o_h = out_head_stride * 2;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window;
    a.sinks = window ? sinks : 0;
    // Rows of a sequence: its new tokens x the query heads of a KV head.  Up to 8, or up to 16 if a batch has no more,
    // are the step kernel's, more the chunk kernel's (a single sequence whole, whatever it brings).  A batch of both takes two
    // launches: 63 single tokens beside a chunk of 1,985 (32 query and 8 KV heads of 128) 198 us, in the
    // chunk kernel alone 222.
    const long long most = (long long)b->max_q * c->dev.G;
    const int few = most <= 16 || c->dev.G > 8 ? 16 : 8;
    cudaStream_t st = (cudaStream_t)stream;
    if (most > few) {
        const bool all = b->num_seqs == 1;
        a.row_lo = all ? 1 : few + 1;
        a.row_hi = 0x7fffffff;
        a.part_o = c->chunk.o;
        a.part_ml = c->chunk.ml;
        a.done = c->chunk.done;
        cudaError_t e = lr::launch_attend_chunk(a, c->maps, c->bf16, c->cfg.format, c->sms, st);
        if (e != cudaSuccess) return cuda_fail(c, e, "attention launch");
        if (all || c->dev.G > few) return LR_OK;
    }
    a.row_lo = 1;
    a.row_hi = (int)std::min<long long>(most, few);
    a.part_o = c->step.o;
    a.part_ml = c->step.ml;
    a.done = c->step.done;
    cudaError_t e = lr::launch_attend_step(a, c->bf16, c->cfg.format, a.row_hi, c->sms, st);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "attention launch");
}

int lr_cache_status(lr_cache *c, void *stream) {
    if (!c) return LR_EINVAL;
    int32_t h = 0;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaMemcpyAsync(&h, c->dev.status, sizeof(int32_t), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess) e = cudaMemsetAsync(c->dev.status, 0, sizeof(int32_t), st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    // a kernel may have given up, whatever error came first: its counts of finished parts start again
    if (e == cudaSuccess && h != LR_OK) {
        e = cudaMemsetAsync(c->chunk.done, 0, 8 * (size_t)c->sms * sizeof(uint32_t), st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return cuda_fail(c, e, "status");
    return h;
}

const char *lr_cache_last_error(const lr_cache *c) { return c ? c->err.c_str() : ""; }

}  // extern "C"
