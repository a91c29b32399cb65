// Attention of many rows over a paged KV cache: chunks of new tokens.
//
// The same one-pass softmax as the step kernel (lr_attend_step.cu), bound by its two matrix
// products instead of the cache's bytes: 4 D operations a (row, token) pair.  A CTA takes 256 rows
// (tokens x query heads of a KV head) against tiles of 128 cached tokens on the tensor cores of sm_103a (tcgen05):
//   S = Q K^T    both operands in shared memory, 128 x 128 fp32 in tensor memory, one for each half of the rows
//   P = exp2(S)  read, exponentiated, rounded to 16 bits and written over S in tensor memory by its threads
//   O += P V     P from tensor memory, V from shared memory, O stays in tensor memory
// Sixteen warps: four a half for the softmax, a thread a row; four that bring K, V and Q to shared
// memory; one thread that issues the products.  The two halves alternate, so that the tensor
// cores work on one while the other's exponentials are taken.
//
// O would have to be scaled whenever a row's maximum rises.  The maximum used is instead left behind
// until it is exceeded by 2^kLag, so after the first tiles O hardly ever moves: any reference
// gives the same quotient, and the weights stay at most 2^kLag.
//
// The batch's tiles are split evenly over the CTAs as in the step kernel, whatever units they belong to.
#include "lr_attend.cuh"

namespace lr {

namespace {

constexpr int kTok = 128;     // tokens of a tile
constexpr int kThreads = 512;
constexpr uint32_t kSpin = 1u << 22;  // polls before a wait gives up

template <int DP, int FMT>
struct Shape {
    static constexpr int kPanel = kTok * 128;                   // 128 rows of 64 16-bit elements
    static constexpr int kTile = kTok * DP * 2;                 // a tile of K or V, or half of Q, in 16 bits
    static constexpr int kStages = FMT == kFmt16 ? 5 : 4;
    // 8-bit codes on their way: 16 bytes a loading thread and slot, as many as the room takes of the
    // 2 * DP / 16 that a tile of K and one of V make
    static constexpr int kSlots = DP == 128 ? 14 : 8;
    static constexpr int kRaw = FMT == kFmt16 ? 0 : kSlots * 128 * 16;
    static constexpr int kQ = 2 * kTile;
    static constexpr int kBytes = kQ + kStages * kTile + kRaw;
    static constexpr int kScales = FMT == kFmt16 ? 0 : 4 * 2 * kTok * 4;
    static constexpr int kSmem = kBytes + kScales + 2 * kTok * 8 + 32 * 8 + (kThreads / 32 + 2) * 8 + 8 * 4;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// ---- barriers in shared memory ----
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n .reg .pred P;\n mbarrier.test_wait.parity.shared::cta.b64 P, [%1], %2;\n selp.u32 %0, 1, 0, P;\n}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
// Waits until the phase of the given parity is over; false if it gives up, or another thread has.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
    for (uint32_t i = 0; i < kSpin; ++i) {
        uint32_t done;
        asm volatile(
            "{\n .reg .pred P;\n mbarrier.try_wait.parity.shared::cta.b64 P, [%1], %2;\n selp.u32 %0, 1, 0, P;\n}"
            : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((i & 1023) == 1023 && *dead) return false;
    }
    *dead = 1;
    return false;
}

// ---- tensor cores ----
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operand descriptor of a 128-byte-swizzled tile: 8-row groups 1,024 bytes apart; `lead`, the distance of
// 64-element panels, matters where the rows are the summed dimension (V).
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead) {
    return (uint64_t)(addr >> 4 & 0x3fff) | (uint64_t)(lead >> 4 & 0x3fff) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 sums of 16-bit products, 128 rows, N columns; `along_n`: B's elements are contiguous along N.
template <bool BF16, int N, bool ALONG_N>
constexpr uint32_t shape_of() {
    return 1u << 4 | (BF16 ? 1u : 0u) << 7 | (BF16 ? 1u : 0u) << 10 | (ALONG_N ? 1u : 0u) << 16 | (N / 8u) << 17 | 8u << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile(
        "{\n .reg .pred P;\n setp.ne.b32 P, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, P;\n}" ::"r"(d), "l"(a),
        "l"(b), "r"(shape), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile(
        "{\n .reg .pred P;\n setp.ne.b32 P, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, P;\n}" ::"r"(d), "r"(a),
        "l"(b), "r"(shape), "r"((uint32_t)add)
        : "memory");
}
// 32 columns of the warp's 32 lanes of tensor memory, a lane a thread.
__device__ __forceinline__ void tm_load(float *r, uint32_t addr) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
          "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
          "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
          "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
__device__ __forceinline__ void tm_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_store(uint32_t addr, const uint32_t *u) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]),
        "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]),
        "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]),
        "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]), "r"(u[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)),
          "l"(reinterpret_cast<unsigned long long &>(c)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void shared_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int DP>
__device__ __forceinline__ uint32_t swizzled(int row, int chunk) {  // byte offset of a 16-byte chunk in a tile
    return (chunk >> 3) * (kTok * 128) + row * 128 + ((chunk ^ row) & 7) * 16;
}

// A row of O in which 32 columns from `col` came out with infinities or NaN (`bad`: which): tokens that the row
// does not see have weight zero, but zero times a value that is not finite is not zero.  The columns
// in which the row sees such a value itself get the sum of those; the others are summed again over what
// it sees.  16-bit caches only (8-bit codes are finite, and their scales are kept from hidden weights).
template <bool BF16>
__device__ __noinline__ void mend(const AttendLaunch &a, const Unit &u, int j0, int j1, int row, int pos, float mref, int col, float *o) {
    const CacheDev &c = a.c;
    const int gr = u.qt * 256 + row, t = quot(gr, c.div_g), hd = u.h * c.G + gr - t * c.G;
    const uint32_t *const q = reinterpret_cast<const uint32_t *>(a.q + (int64_t)(u.q0 + t) * a.q_t + (int64_t)hd * a.q_h);
    for (int d = 0; d < 32; ++d) {
        if (fabsf(o[d]) < INFINITY || col + d >= c.D) continue;
        float seen = 0.0f, sum = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {  // first only the values that are not finite
            if (pass == 1 && seen != 0.0f) break;
            for (int j = j0; j < j1; ++j) {
                const int base = (j < u.ns ? j : u.wf + j - u.ns) * kTok;
                for (int i = base; i < base + kTok; ++i) {
                    if (!visible(pos, i, a.window, a.sinks)) continue;
                    int place;
                    const int64_t blk = block_of(c, a.b, u.s, i, place);
                    if (blk < 0) continue;
                    const int64_t at = blk * c.sb + place * c.st + u.h * c.sh;
                    const uint32_t w = *reinterpret_cast<const uint16_t *>(c.v + at + (col + d) * 2);
                    const float v = unpack16<BF16>(w).x;
                    if (pass == 0) {
                        if (!(fabsf(v) < INFINITY)) seen += v;
                        continue;
                    }
                    const uint32_t *const k = reinterpret_cast<const uint32_t *>(c.k + at);
                    float s = 0.0f;
                    for (int e = 0; e < c.D / 2; ++e) {
                        const float2 x = unpack16<BF16>(q[e]), y = unpack16<BF16>(k[e]);
                        s = fmaf(x.x, y.x, fmaf(x.y, y.y, s));
                    }
                    const float p = exp2_fast(s * a.scale_log2 - mref);
                    sum = fmaf(unpack16<BF16>(pack16<BF16>(p, 0.0f)).x, v, sum);
                }
            }
        }
        o[d] = seen != 0.0f ? seen : sum;
    }
}

template <bool BF16, int FMT, int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attend_chunk(const __grid_constant__ AttendLaunch a) {
    using S = Shape<DP, FMT>;
    constexpr int kStages = S::kStages;
    constexpr float kLag = BF16 ? 8.0f : 4.0f;
    // fp16 weights that carry 8-bit scales: lifted from fp16's subnormal numbers (scales are at most
    // 65504/127 = 516 and weights 2^kLag = 16, so 4 times them stays below 65504)
    constexpr float kLift = FMT != kFmt16 && !BF16 ? 4.0f : 1.0f;
    // (no static shared memory, so that the tiles start where the swizzle's 1,024-byte pattern does)
    extern __shared__ __align__(1024) char smem[];
    char *const tiles = smem + S::kQ;
    char *const raw = tiles + kStages * S::kTile;
    float *const scales = reinterpret_cast<float *>(smem + S::kBytes);                                    // [4][K, V][token]
    int64_t *const places = reinterpret_cast<int64_t *>(smem + S::kBytes + S::kScales);                   // [2][token]
    uint64_t *const bars = reinterpret_cast<uint64_t *>(places + 2 * kTok);
    long long *const scratch = reinterpret_cast<long long *>(bars + 32);
    int *const s_bad = reinterpret_cast<int *>(scratch + kThreads / 32 + 2);                              // [4]
    int *const s_last = s_bad + 4, &s_dead = s_bad[6];                                                    // [2], one
    uint32_t &s_tmem = *reinterpret_cast<uint32_t *>(s_bad + 7);
    const uint32_t b0 = smem_addr(bars);
    // (the barriers: how many arrive, who)
    const uint32_t q_full = b0, q_free = b0 + 8, kv_full = b0 + 16, kv_free = kv_full + 8 * kStages, s_full = kv_free + 8 * kStages,
                   p_full = s_full + 16, o_full = p_full + 16, o_free = o_full + 16, sc_full = o_free + 16, ended = sc_full + 32;
    static_assert(2 + 2 * kStages + 8 + 4 + 1 <= 32, "barriers");
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const CacheDev &c = a.c;

    chain_wait();
    Cursor<256, kTok> cu;
    Share sh;
    if (!take_share<256, kTok, kThreads>(a, cu, sh, scratch)) {
        chain_next();
        return;
    }
    const int count = (int)(sh.x1 - sh.x0);
    if (tid == 0) {
        bar_init(q_full, 128);
        bar_init(q_free, 1);
        for (int i = 0; i < kStages; ++i) {
            bar_init(kv_full + 8 * i, 128);
            bar_init(kv_free + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(s_full + 8 * i, 1);
            bar_init(p_full + 8 * i, 128);
            bar_init(o_full + 8 * i, 1);
            bar_init(o_free + 8 * i, 128);
        }
        for (int i = 0; i < 4; ++i) bar_init(sc_full + 8 * i, 128);
        bar_init(ended, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
        s_dead = 0;
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tm = s_tmem;
    volatile int *const dead = &s_dead;

    if (warp < 8) {
        // ================= softmax: a thread a row =================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int half = warp / 4, r = tid;  // row of the unit
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tm + half * 128 + lanes, to = tm + 256 + half * 128 + lanes;
        uint32_t n_s = 0, n_o = 0;
        bool ok = true;
        // (a wait that gave up leaves `ok` false: the rest is walked through without waiting, the barriers between
        // the threads of the CTA kept)
        for (int x = 0, frag = 0; x < count; ++frag) {
            const Unit &u = cu.u;
            const int n = min(u.nt - cu.j, count - x);
            if (half == 1 && u.rows <= 128) {
                x += n;
                if (x < count) {
                    cu.j += n - 1;
                    cu.next(a);
                }
                continue;
            }
            const int gr = u.qt * 256 + r, t = quot(gr, c.div_g);
            const bool real = r < u.rows;
            const int pos = real ? u.kv - u.ql + t : -1;
            // positions of the half's first and last row
            const int f0 = u.qt * 256 + half * 128, f1 = u.qt * 256 + min(u.rows, half * 128 + 128) - 1;
            const int lo = u.kv - u.ql + quot(f0, c.div_g), hi = u.kv - u.ql + quot(f1, c.div_g);
            float mref = -INFINITY;  // the maximum that the weights refer to, times scale * log2(e)
            float2 l2 = make_float2(0.0f, 0.0f);
            const int j0 = cu.j;
            for (int j = 0; j < n; ++j) {
                const int tile = j0 + j, base = (tile < u.ns ? tile : u.wf + tile - u.ns) * kTok;
                const int slot = (x + j) & 3;
                // (the scores first: a half that skips units may be ahead of the scales' barrier by a phase)
                ok = ok && bar_wait(s_full + 8 * half, n_s & 1, dead) && bar_wait(sc_full + 8 * slot, (x + j) >> 2 & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++n_s;
                after_sync();
                float s[kTok];
#pragma unroll
                for (int k = 0; k < kTok; k += 32) tm_load(s + k, ts + k);
                tm_load_wait();
                const float *const ks = scales + slot * 2 * kTok, *const vs = ks + kTok;
                if constexpr (FMT != kFmt16) {
#pragma unroll
                    for (int k = 0; k < kTok; k += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(ks + k);
                        s[k] *= f.x;
                        s[k + 1] *= f.y;
                        s[k + 2] *= f.z;
                        s[k + 3] *= f.w;
                    }
                }
                const bool masked = base + kTok - 1 > lo || (a.window > 0 && base <= hi - a.window && base + kTok > a.sinks);
                if (masked) {
                    const int top = pos - base, low = a.window > 0 ? pos - a.window - base : -1, sink = a.sinks - base;
#pragma unroll
                    for (int k = 0; k < kTok; ++k)
                        if (!(k <= top && (k > low || k < sink))) s[k] = -INFINITY;
                }
                float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int k = 4; k < kTok; k += 4)
#pragma unroll
                    for (int z = 0; z < 4; ++z) mx[z] = fmaxf(mx[z], s[k + z]);
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
                const bool raise = top > mref + kLag;  // (from -inf: any number)
                if (__any_sync(0xffffffffu, raise)) {
                    const float f = raise ? exp2_fast(mref - top) : 1.0f;  // 0 where nothing was seen yet
                    if (raise) mref = top;
                    l2 = mul2(l2, make_float2(f, f));
                    if (j > 0) {
                        // the sums that the products so far have left: they are done, since this tile's scores come after them
#pragma unroll
                        for (int k = 0; k < DP; k += 32) {
                            float o[32];
                            tm_load(o, to + k);
                            tm_load_wait();
#pragma unroll
                            for (int z = 0; z < 32; ++z) o[z] *= f;
                            tm_store(to + k, reinterpret_cast<uint32_t *>(o));
                        }
                    }
                }
                const float neg = mref == -INFINITY ? 0.0f : -mref;
                const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), neg2 = make_float2(neg, neg);
                uint32_t p[kTok / 2];
#pragma unroll
                for (int k = 0; k < kTok; k += 4) {
                    float2 e = fma2(make_float2(s[k], s[k + 1]), sc2, neg2), g = fma2(make_float2(s[k + 2], s[k + 3]), sc2, neg2);
                    e.x = exp2_fast(e.x);
                    e.y = exp2_fast(e.y);
                    g.x = exp2_fast(g.x);
                    g.y = exp2_fast(g.y);
                    l2 = add2(l2, add2(e, g));
                    if constexpr (FMT != kFmt16) {
                        const float4 f = *reinterpret_cast<const float4 *>(vs + k);
                        e = mul2(e, make_float2(f.x * kLift, f.y * kLift));
                        g = mul2(g, make_float2(f.z * kLift, f.w * kLift));
                        if (masked) {  // a scale that is not finite stays away from a weight that the mask takes
                            if (s[k] == -INFINITY) e.x = 0.0f;
                            if (s[k + 1] == -INFINITY) e.y = 0.0f;
                            if (s[k + 2] == -INFINITY) g.x = 0.0f;
                            if (s[k + 3] == -INFINITY) g.y = 0.0f;
                        }
                    }
                    p[k / 2] = pack16<BF16>(e.x, e.y);
                    p[k / 2 + 1] = pack16<BF16>(g.x, g.y);
                }
                tm_store(ts, p);
                tm_store(ts + 32, p + 32);
                tm_store_wait();
                if (s_bad[slot]) l2.x = __uint_as_float(0x7fffffffu);
                before_sync();
                bar_arrive(p_full + 8 * half);
            }
            // ---- the unit ends here, for this CTA ----
            ok = __all_sync(0xffffffffu, ok && bar_wait(o_full + 8 * half, n_o & 1, dead));
            ++n_o;
            after_sync();
            const float l = l2.x + l2.y;
            const long long u0 = sh.x0 + x - j0, u1 = u0 + u.nt;
            const bool whole = u0 >= sh.x0 && u1 <= sh.x1;
            const int hd = u.h * c.G + gr - t * c.G;
            const int64_t slot = whole ? 0 : slot_of(sh, blockIdx.x, u0);
            char *const po = a.out + (int64_t)(u.q0 + t) * a.o_t + (int64_t)hd * a.o_h;
            float *const pw = a.part_o + (slot * 256 + r) * 128;
            const float inv = l == 0.0f ? 0.0f : 1.0f / (l * kLift);
#pragma unroll
            for (int k = 0; k < DP; k += 32) {
                if (!ok) break;
                float o[32];
                __syncwarp();
                tm_load(o, to + k);
                tm_load_wait();
                if constexpr (FMT == kFmt16) {
                    bool bad = false;
#pragma unroll
                    for (int z = 0; z < 32; ++z) bad |= !(fabsf(o[z]) < INFINITY);
                    if (bad && real && l == l) {
                        float y[32];
#pragma unroll
                        for (int z = 0; z < 32; ++z) y[z] = o[z];
                        mend<BF16>(a, u, j0, j0 + n, r, pos, mref == -INFINITY ? 0.0f : mref, k, y);
#pragma unroll
                        for (int z = 0; z < 32; ++z) o[z] = y[z];
                    }
                }
                if (whole && real) {
#pragma unroll
                    for (int z = 0; z < 32; z += 8)
                        if (k + z < c.D)
                            *reinterpret_cast<uint4 *>(po + (k + z) * 2) =
                                make_uint4(pack16<BF16>(o[z] * inv, o[z + 1] * inv), pack16<BF16>(o[z + 2] * inv, o[z + 3] * inv),
                                           pack16<BF16>(o[z + 4] * inv, o[z + 5] * inv), pack16<BF16>(o[z + 6] * inv, o[z + 7] * inv));
                } else if (real) {
#pragma unroll
                    for (int z = 0; z < 32; z += 4) *reinterpret_cast<float4 *>(pw + k + z) = make_float4(o[z], o[z + 1], o[z + 2], o[z + 3]);
                }
            }
            __syncwarp();
            before_sync();
            bar_arrive(o_free + 8 * half);
            if (real && ok) {
                if (!whole) a.part_ml[slot * 256 + r] = make_float2(mref, l);
                else if (a.lse) a.lse[(int64_t)(u.q0 + t) * c.Hq + hd] = l == 0.0f ? -INFINITY : (mref + log2f(l)) * 0.69314718f;
            }
            if (!whole) {
                // both halves, or the one that has rows
                const int threads = u.rows > 128 ? 256 : 128;
                const int c0 = cta_of(sh, u0), c1 = cta_of(sh, u1 - 1);
                __threadfence();
                named_sync(2, threads);
                if (tid == 0) {
                    const bool last = atomicAdd(a.done + c0, 1u) == (uint32_t)(c1 - c0);
                    if (last) a.done[c0] = 0;
                    s_last[frag != 0] = last;  // (only a CTA's first and last units are shared)
                }
                named_sync(2, threads);
                if (s_last[frag != 0]) {  // join the parts, in the order of the CTAs whichever came last: a warp a row
                    __threadfence();
                    constexpr int kLanes = DP / 4;
                    for (int q = tid / kLanes; q < u.rows; q += threads / kLanes) {
                        const int d = tid % kLanes * 4;
                        float mm = -INFINITY, ll = 0.0f;
                        for (int k = c0; k <= c1; ++k) mm = fmaxf(mm, __ldcg(&a.part_ml[(int64_t)slot_of(sh, k, u0) * 256 + q].x));
                        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        for (int k = c0; k <= c1; ++k) {
                            const int64_t at = (int64_t)slot_of(sh, k, u0) * 256 + q;
                            const float2 ml = __ldcg(a.part_ml + at);
                            const float f = ml.x == -INFINITY ? 0.0f : exp2_fast(ml.x - mm);
                            const float4 w = __ldcg(reinterpret_cast<const float4 *>(a.part_o + at * 128 + d));
                            ll += ml.y == 0.0f ? 0.0f : ml.y * f;
                            if (ml.x == -INFINITY && ml.y == 0.0f) continue;  // saw nothing
                            acc.x += w.x * f;
                            acc.y += w.y * f;
                            acc.z += w.z * f;
                            acc.w += w.w * f;
                        }
                        const int g2 = u.qt * 256 + q, t2 = quot(g2, c.div_g), h2 = u.h * c.G + g2 - t2 * c.G;
                        const float iv = ll == 0.0f ? 0.0f : 1.0f / (ll * kLift);
                        if (d < c.D)
                            *reinterpret_cast<uint2 *>(a.out + (int64_t)(u.q0 + t2) * a.o_t + (int64_t)h2 * a.o_h + d * 2) =
                                make_uint2(pack16<BF16>(acc.x * iv, acc.y * iv), pack16<BF16>(acc.z * iv, acc.w * iv));
                        if (a.lse && d == 0)
                            a.lse[(int64_t)(u.q0 + t2) * c.Hq + h2] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
                    }
                }
            }
            x += n;
            if (x < count) {
                cu.j += n - 1;
                cu.next(a);
            }
        }
    } else if (warp < 12) {
        // ================= K, V and Q to shared memory =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        const int i = tid - 256;
        uint32_t item = 0, frag = 0;
        bool ok = true;
        // 16-bit copies complete in order: the barriers of the last two groups wait for theirs
        uint32_t w0 = 0, w1 = 0;
        auto landed = [&](uint32_t bar) {
            copy_commit();
            if (w1) {
                copy_wait<2>();
                shared_to_async();
                bar_arrive(w1);
            }
            w1 = w0;
            w0 = bar;
        };
        auto drain = [&]() {
            copy_wait<0>();
            shared_to_async();
            if (w1) bar_arrive(w1);
            if (w0) bar_arrive(w0);
            w0 = w1 = 0;
        };
        // where token i of the tile at cursor p is, with its scales
        struct Found {
            int64_t off;
            float ks, vs;
            bool bad;
        };
        auto look = [&](const Cursor<256, kTok> &p) {
            Found f{-1, 0.0f, 0.0f, false};
            const int t = p.base() + i;
            if (t > p.u.hi || (a.window > 0 && t <= p.u.lo - a.window && t >= a.sinks)) return f;
            int place;
            const int64_t blk = block_of(c, a.b, p.u.s, t, place);
            if (blk < 0) {
                f.bad = true;
                report(c.status, kEInval);
                return f;
            }
            f.off = blk * c.sb + place * c.st + p.u.h * c.sh;
            if constexpr (FMT != kFmt16) {
                const int64_t so = blk * c.ssb + place * c.sst + p.u.h * c.ssh;
                f.ks = __ldg(c.ks + so);
                f.vs = __ldg(c.vs + so);
            }
            return f;
        };
        // the copies of tile x of K (y = 0) or V of the places in slot x & 1
        constexpr int CH = FMT == kFmt16 ? DP / 8 : DP / 16, kStep = 128 / CH, kIts = kTok / kStep;
        const int ch = i % CH, r0 = i / CH;
        const bool in = ch * (FMT == kFmt16 ? 8 : 16) < c.D;
        auto queries = [&](const Unit &u) {
            constexpr int QC = DP / 8, QS = 128 / QC;
            const int qc = i % QC;
            for (int r = i / QC; r < 256; r += QS) {
                const int gr = u.qt * 256 + r, t = quot(gr, c.div_g), hd = u.h * c.G + gr - t * c.G;
                const bool real = r < u.rows && qc * 8 < c.D;
                const int64_t at = real ? (int64_t)(u.q0 + t) * a.q_t + (int64_t)hd * a.q_h + qc * 16 : 0;
                copy16(smem_addr(smem + r / 128 * S::kTile) + swizzled<DP>(r % 128, qc), a.q + at, real);
            }
        };
        auto put = [&](int x, const Found &f) {
            places[(x & 1) * kTok + i] = f.off;
            if constexpr (FMT != kFmt16) {
                scales[(x & 3) * 2 * kTok + i] = f.ks;
                scales[(x & 3) * 2 * kTok + kTok + i] = f.vs;
            }
            const unsigned any = __ballot_sync(0xffffffffu, f.bad);
            if (lane == 0 && any) s_bad[x & 3] = 1;
        };
        // stage of the next item, free to be written
        auto stage = [&]() {
            const uint32_t st = item % kStages, round = item / kStages;
            if (round > 0 && ok) {
                if constexpr (FMT == kFmt16) {
                    // a thread that has to wait hands over what it has copied first
                    if (!bar_test(kv_free + 8 * st, (round - 1) & 1)) drain();
                }
                ok = bar_wait(kv_free + 8 * st, (round - 1) & 1, dead);
            }
            return st;
        };
        // 8-bit codes: copy number n of this thread (kIts an item, K and V in turn) of the tile in places slot `at`
        uint32_t ahead = 0;  // copies requested
        auto request = [&](bool any) {
            const uint32_t it = ahead / kIts, k = ahead % kIts;
            if (any) {
                const int64_t off = places[(it >> 1 & 1) * kTok + r0 + k * kStep];
                const bool have = in && off >= 0;
                copy16(smem_addr(raw + (ahead % S::kSlots * 128 + i) * 16), (it & 1 ? c.v : c.k) + (have ? off + ch * 16 : 0), have);
            }
            copy_commit();
            ++ahead;
        };
        if (i < 4) s_bad[i] = 0;
        named_sync(1, 128);
        put(0, look(cu));
        named_sync(1, 128);
        if constexpr (FMT != kFmt16) {
            static_assert(FMT == kFmt16 || S::kSlots <= 2 * kIts, "the first requests are the first tile's");
            for (int k = 0; k < S::kSlots; ++k) request(true);
        }
        for (int x = 0; x < count; ++x) {  // (cu stands at tile x, then at x + 1)
            bar_arrive(sc_full + 8 * (x & 3));  // the tile's scales and flag
            if (x == 0 || cu.j == 0) {
                if constexpr (FMT == kFmt16) drain();
                if (frag > 0 && ok) ok = bar_wait(q_free, (frag - 1) & 1, dead);
                queries(cu.u);
                if constexpr (FMT == kFmt16) {
                    landed(q_full);
                } else {
                    copy_commit();
                    copy_wait<0>();
                    shared_to_async();
                    bar_arrive(q_full);
                }
                ++frag;
            }
            const bool more = x + 1 < count;
            Found f{-1, 0.0f, 0.0f, false};
            if (more) {
                cu.next(a);
                f = look(cu);
            }
            if constexpr (FMT == kFmt16) {
                for (int y = 0; y < 2; ++y, ++item) {
                    const uint32_t st = stage();
                    const uint32_t to = smem_addr(tiles + st * S::kTile);
                    const char *const from = y ? c.v : c.k;
#pragma unroll
                    for (int k = 0; k < kIts; ++k) {
                        const int r = r0 + k * kStep;
                        const int64_t off = places[(x & 1) * kTok + r];
                        const bool have = in && off >= 0;
                        copy16(to + swizzled<DP>(r, ch), from + (have ? off + ch * 16 : 0), have);
                    }
                    landed(kv_full + 8 * st);
                }
            }
            // the next tile's places (8-bit: before this tile's codes are taken, in whose room its own are requested)
            if (i == 0) s_bad[(x + 1) & 3] = 0;
            named_sync(1, 128);
            if (more) put(x + 1, f);
            named_sync(1, 128);
            if constexpr (FMT != kFmt16) {
                for (int y = 0; y < 2; ++y, ++item) {
                    const uint32_t st = stage();
                    const uint32_t to = smem_addr(tiles + st * S::kTile);
#pragma unroll 2
                    for (int k = 0; k < kIts; ++k) {
                        const int r = r0 + k * kStep;
                        const uint32_t at = smem_addr(raw + ((item * kIts + k) % S::kSlots * 128 + i) * 16);
                        copy_wait<S::kSlots - 1>();
                        uint32_t w[4], v[8];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            v[2 * z] = from_codes<BF16, FMT>(w[z], 0, 1);
                            v[2 * z + 1] = from_codes<BF16, FMT>(w[z], 2, 3);
                        }
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + swizzled<DP>(r, 2 * ch)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + swizzled<DP>(r, 2 * ch + 1)), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
                        // the copy that takes this slot next is of this tile's V or of the next tile
                        request(ahead / (2 * kIts) <= (uint32_t)x + (more ? 1 : 0));
                    }
                    shared_to_async();
                    bar_arrive(kv_full + 8 * st);
                }
            }
        }
        if constexpr (FMT == kFmt16) drain();
        copy_wait<0>();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 12 && lane == 0) {
            // ================= products =================
            constexpr uint32_t kQK = shape_of<BF16, kTok, false>(), kPV = shape_of<BF16, DP, true>();
            const uint32_t sq = smem_addr(smem), sk = smem_addr(tiles);
            uint32_t item = 0, n_p[2] = {0, 0}, n_o[2] = {0, 0};
            bool ok = true;
            auto scores = [&](int h, uint32_t st) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t at = (k / 4) * S::kPanel + (k % 4) * 32;
                    mma_ss(tm + h * 128, operand(sq + h * S::kTile + at, 16), operand(sk + st * S::kTile + at, 16), kQK, k > 0);
                }
                commit(s_full + 8 * h);
            };
            auto full = [&](uint32_t it) { return bar_wait(kv_full + 8 * (it % kStages), it / kStages & 1, dead); };
            for (int x = 0, frag = 0; x < count && ok; ++frag) {
                const int n = min(cu.u.nt - cu.j, count - x), nh = cu.u.rows > 128 ? 2 : 1;
                ok = bar_wait(q_full, frag & 1, dead) && full(item);
                if (!ok) break;
                after_sync();
                for (int h = 0; h < nh; ++h) scores(h, item % kStages);
                commit(kv_free + 8 * (item % kStages));
                if (n == 1) commit(q_free);
                ++item;
                for (int j = 0; j < n && ok; ++j) {
                    const bool more = j + 1 < n;
                    const uint32_t sv = item % kStages, sk1 = (item + 1) % kStages;
                    ok = full(item) && (!more || full(item + 1));
                    for (int h = 0; h < nh && ok; ++h) {
                        ok = bar_wait(p_full + 8 * h, n_p[h] & 1, dead) &&
                             (j > 0 || n_o[h] == 0 || bar_wait(o_free + 8 * h, (n_o[h] - 1) & 1, dead));
                        if (!ok) break;
                        ++n_p[h];
                        after_sync();
#pragma unroll
                        for (int k = 0; k < kTok / 16; ++k)
                            mma_ts(tm + 256 + h * 128, tm + h * 128 + k * 8, operand(sk + sv * S::kTile + k * 2048, S::kPanel), kPV,
                                   j > 0 || k > 0);
                        if (more) {
                            scores(h, sk1);
                        } else {
                            commit(o_full + 8 * h);
                            ++n_o[h];
                        }
                    }
                    if (!ok) break;
                    commit(kv_free + 8 * sv);
                    if (more) {
                        commit(kv_free + 8 * sk1);
                        if (j + 2 == n) commit(q_free);
                    }
                    item += more ? 2 : 1;
                }
                x += n;
                if (x < count) {
                    cu.j += n - 1;
                    cu.next(a);
                }
            }
            if (!ok) {  // what was issued ends before its memory is given back
                commit(ended);
                for (uint32_t i = 0; i < kSpin && !bar_test(ended, 0); ++i) {
                }
            }
        }
        __syncwarp();
    }
    __syncthreads();
    if (warp == 12) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
        if (lane == 0 && *dead) report(c.status, kECuda);
    }
    chain_next();
}

using Kernel = void (*)(const AttendLaunch);

template <int FMT, int DP>
Kernel pick_type(bool bf16, size_t &smem) {
    smem = Shape<DP, FMT>::kSmem;
    return bf16 ? k_attend_chunk<true, FMT, DP> : k_attend_chunk<false, FMT, DP>;
}
Kernel pick_kernel(bool bf16, int fmt, int D, size_t &smem) {
    if (D <= 64)
        return fmt == kFmt16 ? pick_type<kFmt16, 64>(bf16, smem)
             : fmt == kFmtE4M3 ? pick_type<kFmtE4M3, 64>(bf16, smem) : pick_type<kFmtInt8, 64>(bf16, smem);
    return fmt == kFmt16 ? pick_type<kFmt16, 128>(bf16, smem)
         : fmt == kFmtE4M3 ? pick_type<kFmtE4M3, 128>(bf16, smem) : pick_type<kFmtInt8, 128>(bf16, smem);
}

}  // namespace

cudaError_t attend_chunk_init() {
    for (int bf16 = 0; bf16 < 2; ++bf16)
        for (int fmt = 0; fmt < 3; ++fmt)
            for (int D = 64; D <= 128; D += 64) {
                size_t smem;
                const Kernel k = pick_kernel(bf16, fmt, D, smem);
                const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
                if (e != cudaSuccess) return e;
            }
    return cudaSuccess;
}

cudaError_t launch_attend_chunk(const AttendLaunch &a, bool bf16, int fmt, int ctas, cudaStream_t st) {
    size_t smem;
    const Kernel k = pick_kernel(bf16, fmt, a.c.D, smem);
    return launch_chained(k, ctas, kThreads, smem, st, a);
}

}  // namespace lr
