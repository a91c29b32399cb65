// Tokens of a paged cache moved together, in place: token kept[i] of a sequence and KV head comes to place start + i.
//
// The lists ascend, so a token never moves up, and what place start + i held is needed by token i or an earlier one alone.
// So a batch of tokens may be written once it and all before it are read, and a later batch is read from places that no
// earlier one writes.  The order holds within a (sequence, KV head) and for each part of a token by itself: K, V, pieces of
// vectors.  A list, or each such part of it where lists are few, is moved by a cluster of CTAs that read a batch, meet,
// and write it, with no other wait.  The meeting orders memory: what is read before it is read before what is written behind it.
//
// What bounds it is the bytes moved, and for short lists the chain list -> block table -> vectors.  Of a long list the chain
// is taken for 512 tokens at once and left in shared memory, with their scales and weights; the vectors then
// follow batch after batch.  A CTA by itself reads the next one before it writes the last one.  A cluster's meeting also waits for the
// writes of the batch before, so it takes batches of twice as much, and the next one's reads run beside those writes (two vectors a thread,
// read ahead as a CTA does: 38 us where four take 34; a meeting that orders no memory, and leaves it to the use of what was read: 32).
// Measured, caches cold: 512 lists of 2,048 tokens (int8, heads of 128, with scales and weights: 480 MB moved) 112 us, 4.3 TB/s; four
// lists of 20,000 tokens in 16 bits 34 us; 2,048 lists of up to 16 tokens 13 us.
#include <algorithm>

#include "lr_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256, kMaxCluster = 16;
constexpr int kAhead = 2, kRun = kThreads * kAhead;  // tokens of a CTA that are looked up together

// Vectors of a batch that a thread moves, where a CTA has both of K and V, or a cluster one of them.
__host__ __device__ constexpr int items(bool both) { return both ? 2 : 4; }

template <int LANES, bool BOTH>
__global__ void __launch_bounds__(kThreads, 4) k_keep(const __grid_constant__ KeepLaunch a) {
    constexpr int kLanes = LANES * (BOTH ? 2 : 1), kItems = items(BOTH), kHeld = BOTH ? 2 : 1;
    __shared__ int4 s_move[kRun];  // block and place of a token, and of where it goes; -1: not moved
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
    // scales and weights move with the first piece
    const bool k_too = (BOTH || !(x & 1)) && piece == 0, v_too = (BOTH || (x & 1)) && piece == 0;
    auto scale_at = [&](int blk, int place) { return (int64_t)blk * c.ssb + place * c.sst + h * c.ssh; };
    auto weight_at = [&](int blk, int place) { return (int64_t)blk * a.wb + place * a.wt + h * a.wh; };
    // The cluster has read what it was to read before it writes.  (Later reads need not wait for these writes: nothing
    // that is read later is written before.)
    auto meet = [&]() {
        if (cl > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    };
    const int run = min(kRun, threads * kAhead) / batch * batch;  // of this CTA; the cluster's CTAs take batches in turn
    for (int64_t r0 = 0; r0 < count; r0 += (int64_t)cl * run) {
        // the token of element e of the run
        auto token = [&](int e) { return r0 + ((int64_t)(e / batch) * cl + rank) * batch + e % batch; };
        int4 m[kAhead];
        float ks[kAhead], vs[kAhead], w[kAhead];
        int src[kAhead], prev[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int e = u * threads + tid;
            const int64_t i = token(e);
            src[u] = e < run && i < count ? __ldg(kept + i) : -1;
            prev[u] = e < run && i < count && i > 0 ? __ldg(kept + i - 1) : -1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int e = u * threads + tid;
            const int64_t i = token(e);
            m[u] = make_int4(-1, 0, -1, 0);
            if (e >= run || i >= count) continue;
            const int dst = start + (int)i;
            if (src[u] < dst || src[u] >= kv || prev[u] >= src[u]) {
                report(c.status, kEInval);
            } else if (src[u] != dst) {
                m[u].x = (int)block_of(c, a.b, s, src[u], m[u].y);
                m[u].z = (int)block_of(c, a.b, s, dst, m[u].w);
                if (m[u].x < 0 || m[u].z < 0) {
                    report(c.status, kEInval);
                    m[u].x = -1;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (u * threads + tid < run) s_move[u * threads + tid] = m[u];
            if (m[u].x >= 0 && c.ks && k_too) ks[u] = c.ks[scale_at(m[u].x, m[u].y)];
            if (m[u].x >= 0 && c.ks && v_too) vs[u] = c.vs[scale_at(m[u].x, m[u].y)];
            if (m[u].x >= 0 && a.w && k_too) w[u] = a.w[weight_at(m[u].x, m[u].y)];
        }
        meet();
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (m[u].x >= 0 && c.ks && k_too) c.ks[scale_at(m[u].z, m[u].w)] = ks[u];
            if (m[u].x >= 0 && c.ks && v_too) c.vs[scale_at(m[u].z, m[u].w)] = vs[u];
            if (m[u].x >= 0 && a.w && k_too) a.w[weight_at(m[u].z, m[u].w)] = w[u];
        }
        // the cluster's batches of the run: as many for each of its CTAs, though the last may have none of their tokens
        const int batches = (int)min((int64_t)(run / batch), (count - r0 + (int64_t)cl * batch - 1) / ((int64_t)cl * batch));
        uint4 v[kHeld][kItems];
        char *to[kHeld][kItems];
        auto read = [&](int n, uint4 (&v)[kItems], char *(&to)[kItems]) {
#pragma unroll
            for (int u = 0; u < kItems; ++u) {
                const int4 at = s_move[n * batch + u * groups + tid / kLanes];
                to[u] = mine && at.x >= 0 ? data + at.z * c.sb + at.w * c.st : nullptr;
                if (to[u]) v[u] = __ldcs(reinterpret_cast<const uint4 *>(data + at.x * c.sb + at.y * c.st));
            }
        };
        auto write = [&](uint4 (&v)[kItems], char *(&to)[kItems]) {
#pragma unroll
            for (int u = 0; u < kItems; ++u)
                if (to[u]) *reinterpret_cast<uint4 *>(to[u]) = v[u];
        };
        if constexpr (BOTH) {
            // (a batch is written after a meeting that all threads come to when they have read the batch behind it)
            read(0, v[0], to[0]);
            for (int n = 0; n < batches; n += 2) {
                if (n + 1 < batches) read(n + 1, v[1], to[1]);
                meet();
                write(v[0], to[0]);
                if (n + 1 >= batches) break;
                if (n + 2 < batches) read(n + 2, v[0], to[0]);
                meet();
                write(v[1], to[1]);
            }
        } else {
            for (int n = 0; n < batches; ++n) {
                read(n, v[0], to[0]);
                meet();
                write(v[0], to[0]);
            }
        }
        if (r0 + (int64_t)cl * run < count) __syncthreads();
    }
    chain_next();
}

}  // namespace

cudaError_t keep_init() {
    cudaError_t e = cudaSuccess;
    for (void (*const k)(const KeepLaunch) : {k_keep<4, false>, k_keep<8, false>, k_keep<16, false>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e;
}

// Lists that fill the GPU take K and V together, a CTA each; fewer are divided into K and V, clusters, and pieces of vectors (64
// bytes at least) while a list is more than a batch.
cudaError_t launch_keep(const KeepLaunch &a, int fmt, int sms, cudaStream_t st) {
    KeepLaunch l = a;
    l.vector = a.c.D * (fmt == kFmt16 ? 2 : 1);
    if (fmt == kFmt16) l.c.ks = l.c.vs = nullptr;
    const long long lists = (long long)a.b.n * a.c.H, room = 4ll * sms;
    int lanes = l.vector <= 64 ? 4 : l.vector <= 128 ? 8 : 16;
    const bool both = lists * 4 > room || (long long)a.cap * 2 * lanes <= kThreads;
    const int kl = lanes * (both ? 2 : 1);
    // (a short list is one or two batches of a smaller CTA: 2,048 lists of up to 16 tokens in 256 threads 14.4 us)
    const int threads = (int)std::min<long long>(kThreads, std::max<long long>(32, ((long long)a.cap * kl / 4 + 31) / 32 * 32));
    l.cluster = 1;
    if (!both) {
        auto batch = [&](int ln) { return (long long)threads / ln * items(false); };
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
