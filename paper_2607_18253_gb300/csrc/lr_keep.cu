// Tokens of a paged cache moved together, in place: token kept[i] of a sequence and KV head comes to place start + i.
//
// The lists ascend, so a token never moves up, and what place start + i held is needed by token i or an earlier one alone.
// So a batch of tokens may be written once it and all before it are read, and a later batch is read from places that no
// earlier one writes.
#include "lr_cache.cuh"

namespace lr {

namespace {

// LPV lanes a vector, 16 bytes a lane; K and V in turn, a CTA a (sequence, KV head, K or V).
constexpr int kThreads = 512, kItems = 4;

template <int LPV>
__global__ void __launch_bounds__(kThreads) k_keep(const __grid_constant__ KeepLaunch a, int vector) {
    const CacheDev &c = a.c;
    const int tid = threadIdx.x, lane = tid % LPV, group = tid / LPV, groups = blockDim.x / LPV;
    chain_wait();
    const bool is_v = blockIdx.x & 1;
    const int list = blockIdx.x >> 1, s = list / c.H, h = list % c.H;
    const int kv = __ldg(a.b.kv_len + s), count = __ldg(a.count + s), start = a.start ? __ldg(a.start + s) : 0;
    const bool bad = kv < 0 || kv > kMaxTokens || (long long)kv > (long long)a.b.max_blocks * c.b || count < 0 || count > a.cap ||
                     (count > 0 && (start < 0 || start > kv - count));
    if (bad || count == 0) {
        if (bad) report(c.status, kEInval);
        chain_next();
        return;
    }
    const int32_t *const kept = a.kept + s * a.kept_s + h * a.kept_h;
    char *const data = is_v ? c.v : c.k;
    float *const scale = is_v ? c.vs : c.ks;
    for (int i0 = 0; i0 < count; i0 += groups * kItems) {
        uint4 x[kItems];
        float sc[kItems], w[kItems];
        int64_t to[kItems];
        int place[kItems];
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int i = i0 + u * groups + group;
            to[u] = -1;
            if (i >= count) continue;
            const int src = __ldg(kept + i), dst = start + i;
            if (src < dst || src >= kv || (i > 0 && __ldg(kept + i - 1) >= src)) {
                report(c.status, kEInval);
                continue;
            }
            if (src == dst) continue;
            int at;
            const int64_t from = block_of(c, a.b, s, src, at), blk = block_of(c, a.b, s, dst, place[u]);
            if (from < 0 || blk < 0) {
                report(c.status, kEInval);
                continue;
            }
            to[u] = blk;
            if (lane * 16 < vector) x[u] = __ldcs(reinterpret_cast<const uint4 *>(data + from * c.sb + at * c.st + h * c.sh + lane * 16));
            if (lane == 0) {
                if (scale) sc[u] = scale[from * c.ssb + at * c.sst + h * c.ssh];
                if (a.w && !is_v) w[u] = a.w[from * a.wb + at * a.wt + h * a.wh];
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (to[u] < 0) continue;
            if (lane * 16 < vector) *reinterpret_cast<uint4 *>(data + to[u] * c.sb + place[u] * c.st + h * c.sh + lane * 16) = x[u];
            if (lane == 0) {
                if (scale) scale[to[u] * c.ssb + place[u] * c.sst + h * c.ssh] = sc[u];
                if (a.w && !is_v) a.w[to[u] * a.wb + place[u] * a.wt + h * a.wh] = w[u];
            }
        }
    }
    chain_next();
}

}  // namespace

cudaError_t launch_keep(const KeepLaunch &a, int fmt, int sms, cudaStream_t st) {
    const int vector = a.c.D * (fmt == kFmt16 ? 2 : 1);
    const unsigned lists = 2u * (unsigned)(a.b.n * a.c.H);
    if (vector <= 64) return launch_chained(k_keep<4>, lists, kThreads, 0, st, a, vector);
    if (vector <= 128) return launch_chained(k_keep<8>, lists, kThreads, 0, st, a, vector);
    return launch_chained(k_keep<16>, lists, kThreads, 0, st, a, vector);
}

}  // namespace lr
