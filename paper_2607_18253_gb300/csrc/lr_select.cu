// The tokens that a cache keeps: of each sequence and KV head the first ones, the most recent ones, and of the rest those
// with the largest weights, ties to the lowest position, in order of position.
//
// A weight becomes a 32-bit key that sorts as it does, a token that is kept in any case the largest.  The key of the last token
// that is kept is found from the top bits down, by counting (11, 11 and 10 bits: three counts of 2,048 bins); the
// tokens above it are kept, and of those equal to it the first ones.  A cluster of CTAs has a list, each a range of its
// positions: the counts and the places of the ranges' tokens are read from one another's shared memory.
#include <algorithm>

#include "lr_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kBins = 2048;
// Keys that a CTA holds in shared memory; further ones are read again for each count.  Of CTAs that are no more than the SMs a
// CTA takes what there is, else what leaves room for three.
constexpr int kHold = 12288, kHoldAlone = 49152;
constexpr int kMaxCluster = 8, kLeast = 2048;  // (positions a CTA, at least, or a list is not divided)
constexpr int kAhead = 8;                      // weights that a thread reads together
constexpr size_t smem_of(int hold) { return (size_t)hold * 4 + 3 * kBins * 4; }

// As `w` sorts: NaN above all, both zeros the same.
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.0f);  // (-0 + 0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The place in CTA `rank`'s shared memory that `p` has in this one's.
__device__ __forceinline__ uint32_t peer(const uint32_t *p, int rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t peer_word(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

__global__ void __launch_bounds__(kThreads) k_select(const __grid_constant__ SelectLaunch a) {
    extern __shared__ __align__(16) uint32_t smem[];
    uint32_t *const bins = smem, *const hold = smem + 3 * kBins;  // [3][kBins], keys
    __shared__ uint32_t s_warp[2 * kWarps], s_bin[2], s_mine[2];
    const int cl = a.cluster;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = cl > 1 ? (int)cluster_rank() : 0;
    const CacheDev &c = a.c;
    chain_wait();
    const int list = blockIdx.x / cl, s = list / c.H, h = list % c.H;
    int kv = __ldg(a.b.kv_len + s), m = a.budget ? __ldg(a.budget + s) : a.cap;
    if (kv < 0 || kv > kMaxTokens || (long long)kv > (long long)a.b.max_blocks * c.b || m < 0 || m > a.cap) {
        report(c.status, kEInval);
        kv = m = 0;
    }
    m = min(m, kv);
    int32_t *const kept = a.kept + (int64_t)list * a.cap;
    if (h == 0 && rank == 0 && tid == 0) a.count[s] = m;
    for (int64_t i = (int64_t)m + rank * kThreads + tid; i < a.cap; i += (int64_t)cl * kThreads) kept[i] = -1;
    if (m == kv || m == 0) {  // (all or none: the whole cluster takes this way)
        for (int64_t i = rank * kThreads + tid; i < m; i += cl * kThreads) kept[i] = (int32_t)i;
        chain_next();
        return;
    }
    // a range of positions a CTA, of it a range a warp, in steps of 32
    const int per = ((kv + cl - 1) / cl + 31) / 32 * 32;
    const int p0 = (int)min((int64_t)kv, (int64_t)rank * per), p1 = (int)min((int64_t)kv, (int64_t)p0 + per);
    auto read = [&](int p) -> uint32_t {
        if (p < a.sinks || p >= kv - a.recent) return 0xffffffffu;
        int place;
        const int64_t blk = block_of(c, a.b, s, p, place);
        if (blk < 0) {
            report(c.status, kEInval);
            return 0u;
        }
        return key_of(a.w[blk * a.wb + place * a.wt + h * a.wh]);
    };
    const int held = a.hold;
    auto key = [&](int p) { return p - p0 < held ? hold[p - p0] : read(p); };

    for (int i = tid; i < 3 * kBins; i += kThreads) bins[i] = 0;
    if (cl > 1) cluster_sync();
    else __syncthreads();
    for (int p = p0 + tid; p < p1; p += kThreads * kAhead) {
        uint32_t k[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) k[i] = p + i * kThreads < p1 ? read(p + i * kThreads) : 0u;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int at = p + i * kThreads;
            if (at >= p1) break;
            if (at - p0 < held) hold[at - p0] = k[i];
            atomicAdd(bins + (k[i] >> 21), 1u);
        }
    }
    uint32_t prefix = 0, need = m;  // the key's bits so far; of the keys that have them, how many are kept
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        uint32_t *const bin = bins + round * kBins;
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, many = round == 2 ? 1024 : kBins;
        if (round > 0) {
            const int above = round == 1 ? 21 : 10;
            for (int p = p0 + tid; p < p1; p += kThreads) {
                const uint32_t k = key(p);
                if (k >> above == prefix >> above) atomicAdd(bin + (k >> shift & (many - 1)), 1u);
            }
        }
        // the cluster's counts come together in its first CTA
        if (rank > 0) {
            __syncthreads();
            for (int i = tid; i < many; i += kThreads)
                if (bin[i]) asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(peer(bin + i, 0)), "r"(bin[i]) : "memory");
        }
        if (cl > 1) cluster_sync();
        else __syncthreads();
        // four bins a thread, from the top: those before the bin that brings the count to `need`
        const int b0 = many - 1 - tid * 4;
        uint32_t v[4] = {0, 0, 0, 0};
        if (b0 >= 0) {
            if (cl > 1)
                asm volatile("ld.shared::cluster.v4.u32 {%3,%2,%1,%0}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(peer(bin + b0 - 3, 0)) : "memory");
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = bin[b0 - i];
        }
        const uint32_t mine = v[0] + v[1] + v[2] + v[3];
        uint32_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        for (int w = 0; w < warp; ++w) incl += s_warp[w];
        uint32_t before = incl - mine;
        if (before < need && need <= incl) {
            int i = 0;
            while (before + v[i] < need) before += v[i++];
            s_bin[0] = b0 - i;
            s_bin[1] = need - before;
        }
        __syncthreads();
        prefix |= s_bin[0] << shift;
        need = s_bin[1];
        __syncthreads();
    }
    // prefix is the last kept token's key now, `need` how many of those equal to it are kept

    const int each = ((p1 - p0 + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int w0 = min(p1, p0 + warp * each), w1 = min(p1, w0 + each);
    uint32_t above = 0, equal = 0;
    for (int p = w0 + lane; p - lane < w1; p += 32) {
        const uint32_t k = p < w1 ? key(p) : 0u;
        above += __popc(__ballot_sync(0xffffffffu, p < w1 && k > prefix));
        equal += __popc(__ballot_sync(0xffffffffu, p < w1 && k == prefix));
    }
    if (lane == 0) {
        s_warp[warp] = above;
        s_warp[kWarps + warp] = equal;
    }
    __syncthreads();
    uint32_t out = 0, eq = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) out += s_warp[w], eq += s_warp[kWarps + w];
    }
    if (cl > 1) {
        if (tid < 2) {
            uint32_t all = 0;
            for (int w = 0; w < kWarps; ++w) all += s_warp[tid * kWarps + w];
            s_mine[tid] = all;
        }
        cluster_sync();
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
            if (r >= rank) break;
            out += peer_word(peer(s_mine, r));
            eq += peer_word(peer(s_mine + 1, r));
        }
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    out += min(eq, need);
    for (int p = w0 + lane; p - lane < w1; p += 32) {
        const uint32_t k = p < w1 ? key(p) : 0u;
        const uint32_t ties = __ballot_sync(0xffffffffu, p < w1 && k == prefix);
        const uint32_t lower = (1u << lane) - 1;
        const bool take = p < w1 && (k > prefix || (k == prefix && eq + __popc(ties & lower) < need));
        const uint32_t all = __ballot_sync(0xffffffffu, take);
        if (take) kept[out + __popc(all & lower)] = p;
        out += __popc(all);
        eq += __popc(ties);
    }
    if (cl > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (no CTA leaves while another reads it)
    chain_next();
}

}  // namespace

cudaError_t select_init() {
    return cudaFuncSetAttribute(k_select, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of(kHoldAlone));
}

cudaError_t launch_select(const SelectLaunch &a, int sms, cudaStream_t st) {
    const long long lists = (long long)a.b.n * a.c.H, longest = std::min((long long)a.b.max_blocks * a.c.b, (long long)kMaxTokens);
    SelectLaunch l = a;
    l.cluster = 1;
    // as many CTAs a list as hold its keys, and more of them for few lists
    while (l.cluster < kMaxCluster && (longest > (long long)kHold * l.cluster || (2 * lists * l.cluster <= 3 * sms && longest >= 2ll * kLeast * l.cluster)))
        l.cluster *= 2;
    const long long each = longest / l.cluster + 64;
    l.hold = (int)std::min(each, (long long)(lists * l.cluster <= sms ? kHoldAlone : kHold));
    return launch_clusters(k_select, (unsigned)(lists * l.cluster), kThreads, smem_of(l.hold), (unsigned)l.cluster, st, l);
}

}  // namespace lr
