// Tokens of a paged cache moved together, in place: token kept[i] of a sequence and KV head comes to place start + i.
//
// The lists ascend, so a token never moves up, and what place start + i held is needed by token i or an earlier one alone.
// So a batch of tokens may be written once it and all before it are read, and a later batch is read from places that no
// earlier one writes.  The order holds within a (sequence, KV head) and for each part of a token by itself: K, V, pieces of
// vectors.  A list, or each such part of it where lists are few, is moved by a cluster of CTAs that read a batch, meet,
// and write it, with no other wait.
//
// What bounds it is the bytes moved, and for short lists the chain list -> block table -> vectors.  The chain is
// taken a batch ahead, by a thread a token, and left in shared memory; of all threads a batch is two times kItems accesses of 16 bytes.
#include <algorithm>

#include "lr_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256, kItems = 4, kMaxCluster = 8;

// LANES lanes a piece of a vector, 16 bytes a lane; BOTH: K and V by the same CTA.
template <int LANES, bool BOTH>
__global__ void __launch_bounds__(kThreads, 5) k_keep(const __grid_constant__ KeepLaunch a) {
    constexpr int kLanes = LANES * (BOTH ? 2 : 1), kBatch = kThreads * kItems / kLanes;
    static_assert(kBatch <= kThreads, "a thread a token");
    __shared__ int4 s_move[2][kBatch];  // block and place of a token, and of where it goes; -1: not moved
    const CacheDev &c = a.c;
    const int tid = threadIdx.x, lane = tid % LANES, cl = a.cluster;
    int x = blockIdx.x / cl;
    const int piece = x % a.pieces;
    x /= a.pieces;
    const bool is_v = BOTH ? tid % kLanes >= LANES : x & 1;
    const int list = BOTH ? x : x >> 1, s = list / c.H, h = list % c.H;
    const int threads = blockDim.x, groups = threads / kLanes, batch = groups * kItems, rank = blockIdx.x % cl;
    const int byte = (piece * LANES + lane) * 16;
    const bool mine = byte < a.vector;
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
    // A thread's token of the batch that begins at i0: block and place of its source and of its place, the first -1 if it is not moved.
    auto look = [&](int i0) {
        int4 m = make_int4(-1, 0, 0, 0);
        const int i = i0 + rank * batch + tid;
        if (i < count) {
            const int src = __ldg(kept + i), dst = start + i, prev = i > 0 ? __ldg(kept + i - 1) : -1;
            const bool good = src >= dst && src < kv && prev < src;
            if (good && src != dst) {
                m.x = (int)block_of(c, a.b, s, src, m.y);
                m.z = (int)block_of(c, a.b, s, dst, m.w);
                if (m.z < 0) m.x = -1;
            }
            if (!good || (src != dst && m.x < 0)) report(c.status, kEInval);
        }
        return m;
    };
    // scales and weight of a token, which its thread moves with the first piece
    const bool k_too = (BOTH || !(x & 1)) && piece == 0, v_too = (BOTH || (x & 1)) && piece == 0;
    auto scale_at = [&](int blk, int place) { return (int64_t)blk * c.ssb + place * c.sst + h * c.ssh; };
    auto weight_at = [&](int blk, int place) { return (int64_t)blk * a.wb + place * a.wt + h * a.wh; };
    if (tid < batch) s_move[0][tid] = look(0);
    __syncthreads();
    int buf = 0;
    for (int i0 = 0; i0 < count; i0 += cl * batch, buf ^= 1) {
        uint4 v[kItems];
        char *to[kItems];
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int4 m = s_move[buf][u * groups + tid / kLanes];
            to[u] = mine && m.x >= 0 ? data + m.z * c.sb + m.w * c.st : nullptr;
            if (to[u]) v[u] = __ldcs(reinterpret_cast<const uint4 *>(data + m.x * c.sb + m.y * c.st));
        }
        float ks, vs, w;
        if (tid < batch) {
            const int4 m = s_move[buf][tid];
            if (m.x >= 0 && c.ks && k_too) ks = c.ks[scale_at(m.x, m.y)];
            if (m.x >= 0 && c.ks && v_too) vs = c.vs[scale_at(m.x, m.y)];
            if (m.x >= 0 && a.w && k_too) w = a.w[weight_at(m.x, m.y)];
        }
        const bool more = i0 + cl * batch < count;
        int4 next;
        if (more && tid < batch) next = look(i0 + cl * batch);
        // (the next batch's reads need not wait for these writes: nothing that it reads is written before)
        if (cl > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
#pragma unroll
        for (int u = 0; u < kItems; ++u)
            if (to[u]) *reinterpret_cast<uint4 *>(to[u]) = v[u];
        if (tid < batch) {
            const int4 m = s_move[buf][tid];
            if (m.x >= 0 && c.ks && k_too) c.ks[scale_at(m.z, m.w)] = ks;
            if (m.x >= 0 && c.ks && v_too) c.vs[scale_at(m.z, m.w)] = vs;
            if (m.x >= 0 && a.w && k_too) a.w[weight_at(m.z, m.w)] = w;
        }
        if (more) {
            if (tid < batch) s_move[buf ^ 1][tid] = next;
            __syncthreads();
        }
    }
    chain_next();
}

}  // namespace

// Lists that fill the GPU take K and V together, a CTA each; fewer are divided into K and V, clusters, and pieces of vectors (64
// bytes at least) while a list is more than a batch.
cudaError_t launch_keep(const KeepLaunch &a, int fmt, int sms, cudaStream_t st) {
    KeepLaunch l = a;
    l.vector = a.c.D * (fmt == kFmt16 ? 2 : 1);
    if (fmt == kFmt16) l.c.ks = l.c.vs = nullptr;
    const long long lists = (long long)a.b.n * a.c.H, room = 2ll * sms;
    int lanes = l.vector <= 64 ? 4 : l.vector <= 128 ? 8 : 16;
    const bool both = lists * 2 > room || (long long)a.cap * 2 * lanes <= kThreads;
    const int kl = lanes * (both ? 2 : 1);
    // (a token a thread at least, so that a short list is one batch)
    const int threads = (int)std::min<long long>(kThreads, std::max<long long>(32, ((long long)a.cap * kl + 31) / 32 * 32));
    l.cluster = 1;
    if (!both) {
        auto batch = [&](int ln) { return (long long)threads / ln * kItems; };
        auto pieces = [&](int ln) { return (l.vector + ln * 16 - 1) / (ln * 16); };
        while (l.cluster < kMaxCluster && lists * 4 * l.cluster <= room && a.cap > batch(lanes) * l.cluster) l.cluster *= 2;
        while (lanes > 4 && lists * 2 * l.cluster * pieces(lanes / 2) <= room && a.cap > batch(lanes) * l.cluster) lanes /= 2;
    }
    l.pieces = (l.vector + lanes * 16 - 1) / (lanes * 16);
    const unsigned grid = (unsigned)(lists * (both ? 1 : 2) * l.pieces * l.cluster);
    void (*const k)(const KeepLaunch) = both ? (lanes == 4 ? k_keep<4, true> : lanes == 8 ? k_keep<8, true> : k_keep<16, true>)
                                             : (lanes == 4 ? k_keep<4, false> : lanes == 8 ? k_keep<8, false> : k_keep<16, false>);
    return launch_clusters(k, grid, threads, 0, l.cluster, st, l);
}

}  // namespace lr
