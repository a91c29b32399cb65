// The tokens that a cache keeps: of each sequence and KV head the first ones, the most recent ones, and of the rest those
// with the largest weights, ties to the lowest position, in order of position.
//
// A weight becomes a 32-bit key that sorts as it does.  The key of the last token that is chosen is found from the top
// byte down, by counting (four counts of 256 bins); the tokens above it are kept, and of those equal to it the first ones.  A cluster of CTAs has a list, each a range of its positions, whose keys it
// holds in shared memory; the counts come together in the first CTA's, and the places of the ranges' tokens are read from one another's.
//
// Short lists are bound by the chain of their steps (block table, weights, four counts, two looks at the keys), many lists by
// the number of such chains that an SM holds.  Measured: 512 lists of 1,024 to 32,768 tokens (8 heads' weights side by side) 68 us, four CTAs
// each; one CTA of 1,024 threads 92, of 512 with keys read again 146.  Four lists of 200,001 tokens, 16 CTAs each, 32 us.
#include <algorithm>

#include "lr_cache.cuh"

namespace lr {

namespace {

constexpr int kBins = 256;
// Keys that a CTA holds in shared memory; further ones are read again for each count.  CTAs that are no more than the SMs have
// 1,024 threads and take what room there is, others have 512 and leave room for four.
constexpr int kHold = 8704, kHoldAlone = 49152;
constexpr int kMaxCluster = 16, kLeast = 2048;  // (positions a CTA, at least, or a list is not divided)
constexpr int kAhead = 8;                       // weights that a thread reads together
constexpr size_t smem_of(int hold) { return (size_t)hold * 4 + 4 * kBins * 4; }

// As `w` sorts: NaN above all, both zeros the same.
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.0f);  // (-0 + 0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
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

template <int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 4 : 1) k_select(const __grid_constant__ SelectLaunch a) {
    constexpr int kWarps = THREADS / 32;
    extern __shared__ __align__(16) uint32_t smem[];
    uint32_t *const bins = smem, *const hold = smem + 4 * kBins;  // [4][kBins], keys
    __shared__ uint32_t s_warp[2 * kWarps], s_bin[2], s_mine[2];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, cl = a.cluster;
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
    // The first tokens, and the last ones: kept in any case.  Between them are the tokens that are chosen from, `need` of them.
    const int head = min(a.sinks, kv), tail = min(a.recent, kv - head), from = head, to = kv - tail;
    uint32_t need = max(0, m - head - tail);
    const int at_tail = head + (int)need;  // where the last ones go (a budget below what is kept in any case takes the first of it)
    for (int64_t i = rank * THREADS + tid; i < a.cap; i += cl * THREADS)
        if (i >= m) kept[i] = -1;
        else if (i < head) kept[i] = (int32_t)i;
        else if (i >= at_tail) kept[i] = to + (int32_t)i - at_tail;
    const int all = to - from;
    if (need == 0 || need == (uint32_t)all) {  // (the whole cluster takes this way)
        if (need)
            for (int i = rank * THREADS + tid; i < all; i += cl * THREADS) kept[head + i] = from + i;
        chain_next();
        return;
    }
    // a range of positions a CTA, of it a range a warp, in steps of 32
    const int per = ((all + cl - 1) / cl + 31) / 32 * 32;
    const int p0 = (int)min((int64_t)to, from + (int64_t)rank * per), p1 = (int)min((int64_t)to, (int64_t)p0 + per);
    const int mid = min(p1, p0 + a.hold);  // (the keys from here on are not held)
    const int32_t *const table = a.b.table + (int64_t)s * a.b.table_stride;
    const float *const weights = a.w + h * a.wh;
    auto read = [&](int p) -> uint32_t {
        const int i = quot(p, c.div_b);
        const int blk = i < a.b.max_blocks ? __ldg(table + i) : -1;
        if ((uint32_t)blk >= (uint32_t)c.nb) {
            report(c.status, kEInval);
            return 0u;
        }
        return key_of(weights[blk * a.wb + (p - i * c.b) * a.wt]);
    };

    for (int i = tid; i < 4 * kBins; i += THREADS) bins[i] = 0;
    if (cl > 1) cluster_sync();
    else __syncthreads();
    for (int p = p0 + tid; p < p1; p += THREADS * kAhead) {
        uint32_t k[kAhead];
        if (p + (kAhead - 1) * THREADS < p1) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) k[i] = read(p + i * THREADS);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (p + i * THREADS < mid) hold[p + i * THREADS - p0] = k[i];
                atomicAdd(bins + (k[i] >> 24), 1u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) k[i] = p + i * THREADS < p1 ? read(p + i * THREADS) : 0u;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (p + i * THREADS >= p1) break;
                if (p + i * THREADS < mid) hold[p + i * THREADS - p0] = k[i];
                atomicAdd(bins + (k[i] >> 24), 1u);
            }
        }
    }
    uint32_t prefix = 0;  // the key's bits so far; of the keys that have them, `need` are kept
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
        uint32_t *const bin = bins + (3 - shift / 8) * kBins;
        if (shift < 24) {
            auto count = [&](uint32_t k) {
                if ((k ^ prefix) >> shift < 256u) atomicAdd(bin + (k >> shift & 255), 1u);
            };
            const int held = mid - p0;
#pragma unroll 4
            for (int i = tid; i < held; i += THREADS) count(hold[i]);
            for (int p = mid + tid; p < p1; p += THREADS) count(read(p));
        }
        // the cluster's counts come together in its first CTA
        if (rank > 0) {
            __syncthreads();
            if (tid < kBins && bin[tid]) asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(peer(bin + tid, 0)), "r"(bin[tid]) : "memory");
        }
        if (cl > 1) cluster_sync();
        else __syncthreads();
        // a bin a thread, from the top: the bin that brings the count to `need`
        if (tid < kBins) {
            const uint32_t mine = cl > 1 ? peer_word(peer(bin + kBins - 1 - tid, 0)) : bin[kBins - 1 - tid];
            uint32_t incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) s_warp[warp] = incl;
            named_sync(1, kBins);
#pragma unroll
            for (int w = 0; w < kBins / 32; ++w)
                if (w < warp) incl += s_warp[w];
            if (incl - mine < need && need <= incl) {
                s_bin[0] = kBins - 1 - tid;
                s_bin[1] = need - (incl - mine);
            }
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
    auto key = [&](int p) { return p < mid ? hold[p - p0] : read(p); };
#pragma unroll 2
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
    if (lane < warp) out = s_warp[lane], eq = s_warp[kWarps + lane];
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        out += __shfl_xor_sync(0xffffffffu, out, o);
        eq += __shfl_xor_sync(0xffffffffu, eq, o);
    }
    if (cl > 1) {
        if (tid < 2) {
            uint32_t sum = 0;
            for (int w = 0; w < kWarps; ++w) sum += s_warp[tid * kWarps + w];
            s_mine[tid] = sum;
        }
        cluster_sync();
        for (int r = 0; r < rank; ++r) {
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
        const uint32_t mask = __ballot_sync(0xffffffffu, take);
        if (take) kept[head + out + __popc(mask & lower)] = p;
        out += __popc(mask);
        eq += __popc(ties);
    }
    if (cl > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (no CTA leaves while another reads it)
    chain_next();
}

}  // namespace

cudaError_t select_init() {
    cudaError_t e = cudaFuncSetAttribute(k_select<1024>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_select<512>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_select<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of(kHoldAlone));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_select<512>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of(kHold));
    return e;
}

cudaError_t launch_select(const SelectLaunch &a, int sms, cudaStream_t st) {
    const long long lists = (long long)a.b.n * a.c.H, longest = std::min((long long)a.b.max_blocks * a.c.b, (long long)kMaxTokens);
    SelectLaunch l = a;
    l.cluster = 1;
    // as many CTAs a list as hold its keys, and more of them for few lists
    while (l.cluster < kMaxCluster && (longest > (long long)kHold * l.cluster || (2 * lists * l.cluster <= sms && longest >= 2ll * kLeast * l.cluster)))
        l.cluster *= 2;
    const bool alone = lists * l.cluster <= sms;
    l.hold = (int)std::min(longest / l.cluster + 64, (long long)(alone ? kHoldAlone : kHold));
    return launch_clusters(alone ? k_select<1024> : k_select<512>, (unsigned)(lists * l.cluster), alone ? 1024 : 512, smem_of(l.hold), (unsigned)l.cluster, st, l);
}

}  // namespace lr
