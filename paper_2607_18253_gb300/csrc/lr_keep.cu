// Tokens of a paged cache moved together, in place: token kept[i] of a sequence and KV head comes to place start + i.
//
// The lists ascend, so a token never moves up, and what place start + i held is needed by token i or an earlier one alone.
// So a batch of tokens may be written once it and all before it are read, and a later batch is read from places that no
// earlier one writes.  The order holds within a (sequence, KV head), K or V, and part of a vector: each such list of parts
// is moved by itself, by a cluster of CTAs that read a batch, meet, and write it, with no other wait.
// Few lists are divided into more parts and larger clusters, so that they fill the GPU.
//
// What bounds it is the bytes moved, and for short lists the chain list -> block table -> vectors.
#include <algorithm>

#include "lr_cache.cuh"

namespace lr {

namespace {

// LANES lanes a part of a vector, 16 bytes a lane; kItems tokens a group of lanes and batch.
constexpr int kThreads = 512, kItems = 4, kMaxCluster = 8;

template <int LANES>
__global__ void __launch_bounds__(kThreads, 2) k_keep(const __grid_constant__ KeepLaunch a) {
    const CacheDev &c = a.c;
    const int tid = threadIdx.x, lane = tid % LANES, cl = a.cluster;
    int x = blockIdx.x / cl;
    const int piece = x % a.pieces;
    x /= a.pieces;
    const bool is_v = x & 1;
    const int list = x >> 1, s = list / c.H, h = list % c.H;
    // the cluster's batch: its CTAs' threads in turn
    const int group = ((int)(blockIdx.x % cl) * (int)blockDim.x + tid) / LANES, groups = cl * (int)blockDim.x / LANES;
    const int byte = (piece * LANES + lane) * 16;
    const bool mine = byte < a.vector, first = piece == 0 && lane == 0;
    chain_wait();
    const int kv = __ldg(a.b.kv_len + s), count = __ldg(a.count + s), start = a.start ? __ldg(a.start + s) : 0;
    const bool bad = kv < 0 || kv > kMaxTokens || (long long)kv > (long long)a.b.max_blocks * c.b || count < 0 || count > a.cap ||
                     (count > 0 && (start < 0 || start > kv - count));
    if (bad || count == 0) {  // (the whole cluster)
        if (bad) report(c.status, kEInval);
        chain_next();
        return;
    }
    const int32_t *const kept = a.kept + s * a.kept_s + h * a.kept_h;
    char *const data = (is_v ? c.v : c.k) + h * c.sh + byte;
    float *const scale = is_v ? c.vs : c.ks, *const weight = is_v ? nullptr : a.w;
    int src[kItems], prev[kItems];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int i = i0 + u * groups + group;
            src[u] = i < count ? __ldg(kept + i) : -1;
            prev[u] = i < count && i > 0 ? __ldg(kept + i - 1) : -1;
        }
    };
    fetch(0);
    for (int i0 = 0; i0 < count; i0 += groups * kItems) {
        uint4 v[kItems];
        float sc[kItems], w[kItems];
        int64_t from[kItems], to[kItems];
        int at[kItems], place[kItems];
        bool move[kItems];
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int i = i0 + u * groups + group, dst = start + i;
            move[u] = i < count;
            if (move[u] && (src[u] < dst || src[u] >= kv || prev[u] >= src[u])) {
                report(c.status, kEInval);
                move[u] = false;
            }
            move[u] = move[u] && src[u] != dst;
            from[u] = to[u] = -1;
            if (move[u]) {
                from[u] = block_of(c, a.b, s, src[u], at[u]);
                to[u] = block_of(c, a.b, s, dst, place[u]);
            }
        }
        if (i0 + groups * kItems < count) fetch(i0 + groups * kItems);
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (!move[u]) continue;
            if (from[u] < 0 || to[u] < 0) {
                report(c.status, kEInval);
                move[u] = false;
                continue;
            }
            if (mine) v[u] = __ldcs(reinterpret_cast<const uint4 *>(data + from[u] * c.sb + at[u] * c.st));
            if (first && scale) sc[u] = scale[from[u] * c.ssb + at[u] * c.sst + h * c.ssh];
            if (first && weight) w[u] = weight[from[u] * a.wb + at[u] * a.wt + h * a.wh];
        }
        // (the next batch's reads need not wait for these writes: nothing that it reads is written before)
        if (cl > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (!move[u]) continue;
            if (mine) *reinterpret_cast<uint4 *>(data + to[u] * c.sb + place[u] * c.st) = v[u];
            if (first && scale) scale[to[u] * c.ssb + place[u] * c.sst + h * c.ssh] = sc[u];
            if (first && weight) weight[to[u] * a.wb + place[u] * a.wt + h * a.wh] = w[u];
        }
    }
    chain_next();
}

}  // namespace

cudaError_t launch_keep(const KeepLaunch &a, int fmt, int sms, cudaStream_t st) {
    KeepLaunch l = a;
    l.vector = a.c.D * (fmt == kFmt16 ? 2 : 1);
    const long long lists = 2ll * a.b.n * a.c.H, room = 2ll * sms;
    // lanes of a whole vector, then of parts of it (64 bytes at least) while the GPU has room and the list more than a batch
    int lanes = l.vector <= 64 ? 4 : l.vector <= 128 ? 8 : 16;
    const int threads = (int)std::min<long long>(kThreads, ((long long)a.cap * lanes / 2 + 31) / 32 * 32 + 32);
    auto batch = [&](int ln) { return (long long)threads / ln * kItems; };
    auto pieces = [&](int ln) { return (l.vector + ln * 16 - 1) / (ln * 16); };
    l.cluster = 1;
    while (l.cluster < kMaxCluster && lists * l.cluster * 2 <= room && a.cap > batch(lanes) * l.cluster) l.cluster *= 2;
    while (lanes > 4 && lists * l.cluster * pieces(lanes / 2) <= room && a.cap > batch(lanes) * l.cluster) lanes /= 2;
    l.pieces = pieces(lanes);
    const unsigned grid = (unsigned)(lists * l.pieces * l.cluster);
    void (*const k)(const KeepLaunch) = lanes == 4 ? k_keep<4> : lanes == 8 ? k_keep<8> : k_keep<16>;
    return launch_clusters(k, grid, threads, 0, l.cluster, st, l);
}

}  // namespace lr
