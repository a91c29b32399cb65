// Host side of the calls on which tokens a paged cache keeps: the weight that they have received, the choice, the move.
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "lr_cache_host.cuh"

using namespace lr;

namespace {

// Weights: a float for each (block, token, head).
const char *bad_weights(const void *w, int64_t block, int64_t token, int64_t head) {
    if (!w || reinterpret_cast<uintptr_t>(w) % 4) return "weights must be a 4-byte aligned device pointer";
    auto good = [](int64_t s) { return s >= 0 && s < (1ll << 56); };
    if (!good(block) || !good(token) || !good(head)) return "strides of weights must be non-negative";
    return nullptr;
}

// (lists of int32; null where there is none)
bool aligned4(std::initializer_list<const void *> lists) {
    for (const void *p : lists)
        if (reinterpret_cast<uintptr_t>(p) % 4) return false;
    return true;
}

const char *bad_lists(const lr_cache *c, const lr_cache_batch *b, int32_t cap) {
    if (cap < 0) return "cap < 0";
    if (b->num_seqs > 0 && (long long)b->num_seqs * c->cfg.num_kv_heads > (1 << 26)) return "too many lists";
    return nullptr;
}

}  // namespace

extern "C" {

int lr_cache_weigh(lr_cache *c, const lr_cache_batch *b, int32_t T, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                   const float *lse, float scale, int32_t window, int32_t sinks, float decay, float *weights, int64_t block_stride,
                   int64_t token_stride, int64_t head_stride, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, T)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (!(std::isfinite(scale) && scale > 0.0f)) return fail(c, LR_EINVAL, "scale must be finite and positive");
    if (!(std::isfinite(decay) && decay >= 0.0f)) return fail(c, LR_EINVAL, "decay must be finite and not negative");
    if (window < 0 || window > kMaxTokens || sinks < 0 || sinks > kMaxTokens) return fail(c, LR_EINVAL, "window and sinks must be in [0, 2^30]");
    if (b->max_q > (1 << 20)) return fail(c, LR_EINVAL, "max_q must be at most 2^20");
    if (T == 0 || b->num_seqs == 0) return LR_OK;
    if (!q || !aligned16(q)) return fail(c, LR_EINVAL, "q must be 16-byte aligned");
    if (!lse || reinterpret_cast<uintptr_t>(lse) % 4) return fail(c, LR_EINVAL, "lse must be a 4-byte aligned device pointer");
    if (!good_stride(q_token_stride, 2) || !good_stride(q_head_stride, 2))
        return fail(c, LR_EINVAL, "strides must be non-negative multiples of 16 bytes");
    if (const char *m = bad_weights(weights, block_stride, token_stride, head_stride)) return fail(c, LR_EINVAL, m);
    WeighLaunch l;
    std::memset(&l, 0, sizeof(l));
    AttendLaunch &a = l.a;
    a.c = c->dev;
    a.b = batch_dev(b, T);
    a.q = static_cast<const char *>(q);
    a.lse = const_cast<float *>(lse);
    a.q_t = q_token_stride * 2;
    a.q_h = q_head_stride * 2;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.part_o = c->weigh.o;
    a.done = c->weigh.done;
    l.w = weights;
    l.wb = block_stride;
    l.wt = token_stride;
    l.wh = head_stride;
    l.decay = decay;
    const double ratio = (double)a.scale_log2 / (double)scale;
    l.lse_log2 = (float)ratio;
    l.lse_log2_rest = (float)(ratio - (double)l.lse_log2);
    cudaError_t e = launch_weigh(l, c->maps, c->bf16, c->cfg.format, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "weigh launch");
}

int lr_cache_select(lr_cache *c, const lr_cache_batch *b, const float *weights, int64_t block_stride, int64_t token_stride,
                    int64_t head_stride, int32_t cap, const int32_t *budget, int32_t sinks, int32_t recent, int32_t *kept,
                    int32_t *count, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, 0, false)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (const char *m = bad_lists(c, b, cap)) return fail(c, LR_EINVAL, m);
    if (sinks < 0 || recent < 0 || (long long)sinks + recent > cap) return fail(c, LR_EINVAL, "sinks and recent must not be negative, and fit into cap");
    if (b->num_seqs == 0) return LR_OK;
    if (const char *m = bad_weights(weights, block_stride, token_stride, head_stride)) return fail(c, LR_EINVAL, m);
    if (!count || (cap > 0 && !kept)) return fail(c, LR_EINVAL, "null kept or count");
    if (!aligned4({kept, count, budget})) return fail(c, LR_EINVAL, "kept, count and budget must be 4-byte aligned");
    SelectLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.c = c->dev;
    a.b = batch_dev(b, 0);
    a.w = weights;
    a.wb = block_stride;
    a.wt = token_stride;
    a.wh = head_stride;
    a.budget = budget;
    a.cap = cap;
    a.sinks = sinks;
    a.recent = recent;
    a.kept = kept;
    a.count = count;
    cudaError_t e = launch_select(a, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "select launch");
}

int lr_cache_keep(lr_cache *c, const lr_cache_batch *b, int32_t cap, const int32_t *kept, int32_t kept_heads, const int32_t *count,
                  const int32_t *start, float *weights, int64_t block_stride, int64_t token_stride, int64_t head_stride, void *stream) {
    if (!c) return LR_EINVAL;
    c->err.clear();
    if (const char *m = bad_batch(b, 0, false)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs > c->cfg.max_seqs) return fail(c, LR_ECAPACITY, "num_seqs exceeds max_seqs");
    if (const char *m = bad_lists(c, b, cap)) return fail(c, LR_EINVAL, m);
    if (kept_heads != 1 && kept_heads != c->cfg.num_kv_heads) return fail(c, LR_EINVAL, "kept_heads must be 1 or num_kv_heads");
    if (weights)
        if (const char *m = bad_weights(weights, block_stride, token_stride, head_stride)) return fail(c, LR_EINVAL, m);
    if (b->num_seqs == 0 || cap == 0) return LR_OK;
    if (!kept || !count) return fail(c, LR_EINVAL, "null kept or count");
    if (!aligned4({kept, count, start})) return fail(c, LR_EINVAL, "kept, count and start must be 4-byte aligned");
    KeepLaunch a;
    std::memset(&a, 0, sizeof(a));
    a.c = c->dev;
    a.b = batch_dev(b, 0);
    a.kept = kept;
    a.kept_s = (int64_t)cap * kept_heads;
    a.kept_h = kept_heads == 1 ? 0 : cap;
    a.count = count;
    a.start = start;
    a.cap = cap;
    a.w = weights;
    a.wb = block_stride;
    a.wt = token_stride;
    a.wh = head_stride;
    cudaError_t e = launch_keep(a, c->cfg.format, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? LR_OK : cuda_fail(c, e, "keep launch");
}

}  // extern "C"
