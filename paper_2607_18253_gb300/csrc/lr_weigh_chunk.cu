// Attention weight that cached tokens have received, from many rows: chunks of new tokens, or the last tokens of prompts.
//
// The formula of lr_weigh.cu on the tensor cores of sm_103a (tcgen05), with the tokens as the products' rows: S = K Q^T is
// 128 tokens by 128 rows of queries in tensor memory, a lane a token, so that a thread takes the exponentials of its token's
// scores and adds them up -- nothing is exchanged between threads, there is no maximum to follow, and the sum's
// order is the rows'.  A unit is a sequence, a KV head and 256 tokens, whose K stays in shared memory while the tiles of
// rows pass: Q is all that moves, for 512 operations a byte.  The two halves of 128 tokens have two buffers of scores
// each, so that the tensor cores work on one while another's exponentials are taken.
// The batch is one line of (unit, tile of rows), cut into equal shares for the CTAs; a unit that is cut is joined by
// the last of its CTAs, in their order.  Of few rows (128 or less a KV head) a unit is one tile, and K's bytes bound it.
//
// Measured (32 query heads on 8 KV heads of 128, 16 bits): 4,096 rows at the end of 32,768 tokens 872 us, 1,180 TFLOP/s.  A tile (256
// tokens x 128 rows) takes 2,140 cycles, of which the products 1,600, where the tensor cores need 1,024: both operands come from shared
// memory, which also takes Q and gives the rows' lse.  The exponentials are 1,170 cycles beside them.  Slower were K in tensor
// memory with tiles of 96 rows (965 us), 16 warps of exponentials (939; with K in tensor memory 1,033), and three of eight
// exponentials as polynomials (1,268); two or four stages of Q or K changed nothing.
// The last 32 tokens of five prompts of 4,096 to 32,768 (128 rows): 49 us, 3.2 TB/s; a unit is 64 KB of K and some
// 5,000 cycles, much of it the walk from unit to unit, which every kind of warp makes, out of a cold instruction cache.
#include "lr_attend.cuh"
#include "lr_tensor.cuh"

namespace lr {

namespace {

constexpr int kThreads = 512, kUnit = 2 * kTok, kRowTile = 128;

// A tile of rows is as many tokens' as 128 holds, whole, so that it is one box of the tensor copy engine (`rt` rows).  The other
// columns of 128 have queries of zero and -inf for -lse, which makes nothing of them where K is finite: zero times K is zero.  Where the
// last column's score is not, the tile takes the way that leaves out what it must.
struct ChunkLaunch {
    WeighLaunch w;
    CacheMaps m;
    CUtensorMap q;
    int32_t q_map, rt;
    FastDiv div_rt;
};

// How K reaches shared memory: a 16-bit cache's by the copy engine, or where blocks are odd 16 bytes a thread; 8-bit codes by
// threads, converted on the way.
enum : int { kTma = 0, kGather = 1, kConvert = 2 };
constexpr int kWeight = 2;  // tiles that a unit's beginning and end take the time of
constexpr int kLeast = 3;   // of a CTA's share

template <int DP>
struct Shape {
    static constexpr int kPanel = kTok * 128, kTile = kTok * DP * 2;
    static constexpr int kKeys = DP == 128 ? 3 : 6, kRows = DP == 128 ? 3 : 4;  // stages of K and Q
    static constexpr int kLess = 8;  // tiles of lse: they are held until the exponentials are taken, Q only for the products
    static constexpr int kBars = 2 * kKeys + 2 * kRows + 2 * kLess + 8 + 1;
    static constexpr int kTiles = (kKeys + kRows) * kTile;
    static constexpr int kSmem = kTiles + kKeys * kTok * 12 + kLess * kRowTile * 4 + 2 * kTok * 8 + kBars * 8 + (kThreads / 32 + 2) * 8 + kLess * 4 + 16;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// A place in the line.
struct Line {
    int s, q0, ql, kv, lo, rows, nq;  // sequence: first new token's position, rows of a KV head, tiles of them
    int ns, wf, nu;                   // units of sinks before the window, the window's first unit, units in all
    int h, u;                         // KV head, unit
    FastDiv div_rt;                   // rows of a tile
    int r0, n;                        // the unit's first tile of rows, and how many
    int j, end;                       // tile of rows from r0 on; the CTA's tiles of the unit end there
    bool last;                        // its last unit
    long long at;                     // where the unit begins

    __device__ __forceinline__ bool load(const WeighLaunch &a) {
        if (!load_seq(a.a, s, q0, ql, kv) || kv == 0) return false;
        lo = kv - ql;
        rows = ql * a.a.c.G;
        nq = quot(rows - 1, div_rt) + 1;
        if (a.decay == 1.0f) nu = tile_count<kUnit>(lo, kv - 1, a.a.window, a.a.sinks, ns, wf);
        else ns = wf = 0, nu = (kv - 1) / kUnit + 1;
        return true;
    }
    __device__ __forceinline__ int base() const { return (u < ns ? u : wf + u - ns) * kUnit; }
    // The unit's tiles of rows that see one of its tokens (one at least, which may see none).
    __device__ __forceinline__ void span(const WeighLaunch &a) {
        const int b = base(), G = a.a.c.G;
        r0 = b > lo ? quot((int)min((long long)(rows - 1), (long long)(b - lo) * G), div_rt) : 0;
        int r1 = nq;
        if (a.a.window > 0 && b >= a.a.sinks) {
            const long long e = ((long long)min(b + kUnit - 1, kv - 1) + a.a.window - lo) * G;  // rows before this one
            r1 = e <= 0 ? 0 : quot((int)min((long long)rows, e) - 1, div_rt) + 1;
        }
        n = max(1, r1 - r0);
    }
    // Tiles of a KV head with the units' weights.
    __device__ __forceinline__ long long cost(const WeighLaunch &a) {
        long long sum = 0;
        u = 0;
        if (a.a.window == 0 && lo >= 0) {  // units that all rows see
            u = min(nu, lo / kUnit + 1);
            sum = (long long)u * (nq + kWeight);
        }
        for (; u < nu; ++u) {
            span(a);
            sum += n + kWeight;
        }
        return sum;
    }
    __device__ __forceinline__ void enter(const WeighLaunch &a, const Share &sh) {
        span(a);
        end = (int)min((long long)n, sh.x1 - at - kWeight);
        last = at + n + 2 * kWeight >= sh.x1;
    }
    __device__ __forceinline__ void next(const WeighLaunch &a, const Share &sh) {  // (not the last)
        j = 0;
        at += n + kWeight;
        if (a.a.window == 0 && u + 1 < nu && (u + 1) * kUnit <= lo) {  // (nearly always: another unit that all rows see)
            ++u;
            end = (int)min((long long)n, sh.x1 - at - kWeight);
            last = at + n + 2 * kWeight >= sh.x1;
            return;
        }
        if (++u == nu) {
            u = 0;
            if (++h == a.a.c.H) {
                h = 0;
                do ++s;
                while (s < a.a.b.n && !load(a));
            }
        }
        enter(a, sh);
    }
    __device__ __forceinline__ int halves() const { return base() + kTok < kv ? 2 : 1; }
    __device__ __forceinline__ bool whole() const { return j == 0 && end == n; }
};

// This CTA's share, with `l` at its first tile; false if it has none.
__device__ __forceinline__ bool take_line(const WeighLaunch &a, Line &l, Share &sh, long long *scratch) {
    long long *const s_sum = scratch, &s_rest = scratch[kThreads / 32], &s_seq = scratch[kThreads / 32 + 1];
    const int n = a.a.b.n, tid = threadIdx.x;
    auto cost_of = [&](int s) -> long long {
        l.s = s;
        return s < n && l.load(a) ? a.a.c.H * l.cost(a) : 0;
    };
    long long all = 0, first = 0, incl = 0, mine = 0;
    for (int base = 0; base < n; base += kThreads) {
        mine = cost_of(base + tid);
        long long t;
        incl = block_sum<kThreads>(mine, s_sum, t);
        all += t;
    }
    if (all == 0) return false;
    sh.all = all;
    sh.ctas = (int)min((long long)gridDim.x, max(all / kLeast, 1ll));
    const int c = blockIdx.x;
    if (c >= sh.ctas) return false;
    sh.x0 = share_start(sh, c);
    sh.x1 = share_start(sh, c + 1);
    for (int base = 0; base < n; base += kThreads) {
        long long t = all;
        if (n > kThreads) {
            mine = cost_of(base + tid);
            incl = block_sum<kThreads>(mine, s_sum, t);
        }
        const long long x = sh.x0 - first;
        if (x < incl && x >= incl - mine) {
            s_seq = base + tid;
            s_rest = x - (incl - mine);
        }
        first += t;
        if (first > sh.x0) break;
    }
    __syncthreads();
    l.s = (int)s_seq;
    l.load(a);
    long long r = s_rest;
    const long long per = l.cost(a);
    l.h = (int)(r / per);
    r -= l.h * per;
    l.u = 0;
    if (a.a.window == 0 && l.lo >= 0) {
        const int full = min(l.nu, l.lo / kUnit + 1);
        l.u = (int)min((long long)full, r / (l.nq + kWeight));
        r -= (long long)l.u * (l.nq + kWeight);
    }
    for (;; ++l.u) {
        l.span(a);
        if (r < l.n + kWeight) break;
        r -= l.n + kWeight;
    }
    l.at = sh.x0 - r;
    l.enter(a, sh);
    l.j = max(0, (int)r - kWeight);
    return l.j < l.end;  // (a share may end in a unit's weight)
}

template <bool BF16, int FMT, int DP, int LOAD>
__global__ void __launch_bounds__(kThreads, 1) k_weigh_chunk(const __grid_constant__ ChunkLaunch in) {
    const WeighLaunch &a = in.w;
    using S = Shape<DP>;
    extern __shared__ __align__(1024) char smem[];
    char *const keys = smem, *const rows = smem + S::kKeys * S::kTile;
    float *const s_less = reinterpret_cast<float *>(smem + S::kTiles);  // [stage][row] -lse * log2(e); -inf: adds nothing
    float *const s_scale = s_less + S::kLess * kRowTile;                // [stage][token] the scores' factor
    int64_t *const s_to = reinterpret_cast<int64_t *>(s_scale + S::kKeys * kTok);  // [stage][token] where its weight is, -1: no place
    int64_t *const s_from = s_to + S::kKeys * kTok;                                // [2][token] where its K is
    uint64_t *const bars = reinterpret_cast<uint64_t *>(s_from + 2 * kTok);
    long long *const scratch = reinterpret_cast<long long *>(bars + S::kBars);
    int *const s_odd = reinterpret_cast<int *>(scratch + kThreads / 32 + 2);  // [stage] a row whose lse is infinite
    int &s_dead = s_odd[S::kLess];
    uint32_t &s_tmem = *reinterpret_cast<uint32_t *>(s_odd + S::kLess + 1);
    uint32_t &s_sent = *reinterpret_cast<uint32_t *>(s_odd + S::kLess + 2);  // tiles of Q, and of K, that the copy engine was asked for
    uint32_t &s_sent_k = *reinterpret_cast<uint32_t *>(s_odd + S::kLess + 3);
    const uint32_t k_full = smem_addr(bars), k_free = k_full + 8 * S::kKeys, q_full = k_free + 8 * S::kKeys, q_free = q_full + 8 * S::kRows,
                   l_full = q_free + 8 * S::kRows, l_free = l_full + 8 * S::kLess, s_full = l_free + 8 * S::kLess, s_free = s_full + 32, ended = s_free + 32;  // scores: [half][buffer]
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const CacheDev &c = a.a.c;

    chain_wait();
    Line l;
    l.div_rt = in.div_rt;
    Share sh;
    if (!take_line(a, l, sh, scratch)) {
        chain_next();
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < S::kKeys; ++i) {
            bar_init(k_full + 8 * i, LOAD == kTma ? 5 : 4);
            bar_init(k_free + 8 * i, 5);
        }
        for (int i = 0; i < S::kRows; ++i) {
            bar_init(q_full + 8 * i, 1);
            bar_init(q_free + 8 * i, 1);
        }
        for (int i = 0; i < S::kLess; ++i) {
            bar_init(l_full + 8 * i, 1);
            bar_init(l_free + 8 * i, 8);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(s_full + 8 * i, 1);
            bar_init(s_free + 8 * i, 4);
        }
        bar_init(ended, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
        s_dead = 0;
        s_sent = s_sent_k = 0;
    }
    for (int i = tid; i < S::kRows * (kRowTile - in.rt) * DP / 8; i += kThreads) {  // rows of Q's stages that no tile fills
        const int r = i / (DP / 8) % (kRowTile - in.rt) + in.rt, st = i / (DP / 8) / (kRowTile - in.rt);
        *reinterpret_cast<uint4 *>(rows + st * S::kTile + swizzled<DP>(r, i % (DP / 8))) = make_uint4(0, 0, 0, 0);
    }
    shared_to_async();
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tm = s_tmem;
    volatile int *const dead = &s_dead;
    uint32_t key = 0, qi = 0;  // tiles of K and of Q so far
    bool ok = true;

    if (warp < 8) {
        // ================= exponentials and sums: a thread a token =================
        const int half = warp / 4, t = tid % kTok;
        const uint32_t ts = tm + half * 256 + ((uint32_t)(warp % 4) << 21);
        uint32_t n_s = 0;  // the half's scores so far
        bool skipped = false;  // the last unit had none of the half's tokens
        for (;; l.next(a, sh)) {
            const int halves = l.halves(), p = l.base() + half * kTok + t;
            const bool on = half < halves, whole = l.whole();
            float f = 0.0f, old = 0.0f;
            int64_t to = -1;
            if (on) {
                // A half that skipped units waited for their rows alone, and may have come here two phases ahead of this stage's barrier, whose
                // parity does not tell them apart.  Its scores of the unit come after their K, and all K before it.
                if (skipped) ok = bar_wait(s_full + 16 * half + 8 * (n_s & 1), n_s >> 1 & 1, dead);
                const uint32_t st = (key + half) % S::kKeys;
                ok = ok && bar_wait(k_full + 8 * st, (key + half) / S::kKeys & 1, dead);
                if (!ok) break;
                f = s_scale[st * kTok + t];
                to = s_to[st * kTok + t];
                bar_arrive_warp(k_free + 8 * st);
                if (whole && to >= 0 && a.decay != 0.0f && p < l.lo) old = a.decay * a.w[to];
            }
            skipped = !on;
            key += halves;
            // the rows that see the token: from the first of its position on, and where a window hides it up to a last
            const int first = p > l.lo ? (int)min((long long)l.rows, (long long)(p - l.lo) * c.G) : 0;
            int end = to < 0 ? 0 : l.rows;
            if (a.a.window > 0 && p >= a.a.sinks) end = (int)min((long long)end, max(0ll, ((long long)p + a.a.window - l.lo) * c.G));
            float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
            const float2 f2 = make_float2(f, f);
            const int j1 = l.end, unit_r0 = l.r0, unit_rows = l.rows;
            for (int j = l.j; j < j1; ++j, ++qi) {
                const uint32_t st = qi % S::kLess;
                ok = bar_wait(l_full + 8 * st, qi / S::kLess & 1, dead);
                if (on) ok = ok && bar_wait(s_full + 16 * half + 8 * (n_s & 1), n_s >> 1 & 1, dead);
                if (!ok) break;
                if (on) {
                    after_sync();
                    const float *const less = s_less + st * kRowTile;
                    const uint32_t from = ts + (n_s & 1) * 128;
                    const int row0 = (unit_r0 + j) * in.rt, some = min(in.rt, unit_rows - row0);
                    // 32 scores of the token; a tile's are summed by themselves first (16,384 rows one after the other are off by 2e-6)
                    float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                    auto add = [&](const float *s, int k0) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 g = *reinterpret_cast<const float4 *>(less + k0 + k);
                            float2 x = fma2(make_float2(s[k], s[k + 1]), f2, make_float2(g.x, g.y));
                            float2 y = fma2(make_float2(s[k + 2], s[k + 3]), f2, make_float2(g.z, g.w));
                            x.x = exp2_fast(x.x);
                            x.y = exp2_fast(x.y);
                            y.x = exp2_fast(y.x);
                            y.y = exp2_fast(y.y);
                            part[0] = add2(part[0], x);
                            part[1] = add2(part[1], y);
                        }
                    };
                    float x[32], y[32];
                    bool all = __all_sync(0xffffffffu, first <= row0 && end >= row0 + in.rt) && !s_odd[st];
                    if (all) {
                        tm_load(x, from + 96);
                        tm_load_wait(x);
                        all = in.rt == kRowTile || __all_sync(0xffffffffu, x[31] * f == 0.0f);
                    }
                    if (all) {
                        tm_load(y, from);
                        add(x, 96);
                        tm_load_wait(y);
                        tm_load(x, from + 32);
                        add(y, 0);
                        tm_load_wait(x);
                        tm_load(y, from + 64);
                        add(x, 32);
                        tm_load_wait(y);
                        before_sync();
                        bar_arrive_warp(s_free + 16 * half + 8 * (n_s & 1));
                        add(y, 64);
                    } else {
                        // (what a row does not see, or is no row of the tile, is left out, whatever it is; the others are summed as above)
                        const int last = min(end, row0 + some);
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            const int k0 = i == 0 ? 96 : i * 32 - 32, r = row0 + k0;
                            if (__all_sync(0xffffffffu, first >= r + 32 || last <= r)) continue;
                            tm_load(x, from + k0);
                            tm_load_wait(x);
#pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                const float g = less[k0 + k], e = exp2_fast(fmaf(x[k], f, g));
                                float &sum_k = k & 1 ? part[k >> 1 & 1].y : part[k >> 1 & 1].x;
                                sum_k += r + k >= first && r + k < last && g != -INFINITY ? e : 0.0f;
                            }
                        }
                        before_sync();
                        bar_arrive_warp(s_free + 16 * half + 8 * (n_s & 1));
                    }
                    sum[0] = add2(sum[0], part[0]);
                    sum[1] = add2(sum[1], part[1]);
                    ++n_s;
                }
                bar_arrive_warp(l_free + 8 * st);
            }
            if (!ok) break;
            // ---- the unit ends here, for this CTA ----
            if (on) {
                float w = (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
                if (whole) {
                    if (to >= 0) a.w[to] = old + w;
                } else {
                    const int c0 = cta_of(sh, l.at + kWeight), c1 = cta_of(sh, l.at + kWeight + l.n - 1);
                    a.a.part_o[(int64_t)slot_of(sh, blockIdx.x, l.at) * kUnit + half * kTok + t] = w;
                    uint32_t before = 0;
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) {
                        before = atomicAdd(a.a.done + c0 * 8 + warp, 1u);
                        if (before == (uint32_t)(c1 - c0)) a.a.done[c0 * 8 + warp] = 0;
                    }
                    before = __shfl_sync(0xffffffffu, before, 0);
                    if (before == (uint32_t)(c1 - c0)) {
                        __threadfence();
                        const int slot0 = slot_of(sh, c0, l.at);
                        w = 0.0f;
#pragma unroll 4
                        for (int k = 0; k <= c1 - c0; ++k)
                            w += __ldcg(a.a.part_o + (int64_t)(k == 0 ? slot0 : 2 * (c0 + k)) * kUnit + half * kTok + t);
                        if (to >= 0) a.w[to] = (a.decay != 0.0f && p < l.lo ? a.decay * a.w[to] : 0.0f) + w;
                    }
                }
            }
            if (l.last) break;
        }
    } else if (warp == 8) {
        // ================= products: the warp waits, one thread issues =================
        const bool one = elect();
        uint32_t n_s[2] = {0, 0};
        for (;; l.next(a, sh)) {
            const int halves = l.halves(), j0 = l.j, j1 = l.end, unit_r0 = l.r0, unit_rows = l.rows;
            for (int j = j0; j < j1 && ok; ++j, ++qi) {
                const uint32_t sq = qi % S::kRows;
                // (a full tile has all 128 columns, of which those of no row are zero)
                const int some = unit_rows - (unit_r0 + j) * in.rt, many = some >= in.rt ? kRowTile : (some + 15) / 16 * 16;
                const uint32_t shape = shape_of<BF16, 0, false>() | (uint32_t)(many / 8) << 17;
                ok = bar_wait(q_full + 8 * sq, qi / S::kRows & 1, dead);
                const uint64_t dq = operand(smem_addr(rows + sq * S::kTile), 16);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (g >= halves || !ok) continue;
                    const uint32_t st = (key + g) % S::kKeys, buf = 16 * g + 8 * (n_s[g] & 1);
                    if (j == j0) ok = bar_wait(k_full + 8 * st, (key + g) / S::kKeys & 1, dead);
                    if (ok && n_s[g] >= 2) ok = bar_wait(s_free + buf, ((n_s[g] >> 1) - 1) & 1, dead);
                    if (!ok) continue;
                    after_sync();
                    if (one) {
                        const uint64_t dk = operand(smem_addr(keys + st * S::kTile), 16);
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            const uint32_t at = (k / 4) * (S::kPanel >> 4) + (k % 4) * 2;  // (descriptors count 16 bytes)
                            mma_ss(tm + g * 256 + (n_s[g] & 1) * 128, dk + at, dq + at, shape, k > 0);
                        }
                        commit(s_full + buf);
                        if (j + 1 == j1) commit(k_free + 8 * st);
                    }
                    __syncwarp();
                    ++n_s[g];
                }
                if (one && ok) commit(q_free + 8 * sq);
                __syncwarp();
            }
            key += halves;
            if (!ok || l.last) break;
        }
    } else if (warp >= 12) {
        // ================= K to shared memory =================
        const int i = tid - 384;
        constexpr int CH = FMT == kFmt16 ? DP / 8 : DP / 16, kStep = 128 / CH, kIts = kTok / kStep;
        const int ch = i % CH, r0 = i / CH;
        const bool in = ch * (FMT == kFmt16 ? 8 : 16) < c.D;
        // copies complete in order: the barriers of the last two tiles wait for theirs
        uint32_t w0 = 0, w1 = 0;
        auto drain = [&]() {
            copy_wait<0>();
            shared_to_async();
            if (w1) bar_arrive_warp(w1);
            if (w0) bar_arrive_warp(w0);
            w0 = w1 = 0;
        };
        struct Found {
            int64_t from, to;  // -1: nothing to read, no place
            float scale;
        };
        // where the thread's token of the tile is; g: half of the unit
        auto look = [&](int g) {
            Found f{-1, -1, a.a.scale_log2};
            const int p = l.base() + g * kTok + i;
            const bool any = !(a.a.window > 0 && p <= l.lo - a.a.window && p >= a.a.sinks);  // (some row sees it)
            if (p >= l.kv || (!any && a.decay == 1.0f)) return f;
            int place;
            const int64_t blk = block_of(c, a.a.b, l.s, p, place);
            if (blk < 0) {  // (a token that no row sees may have no block any more)
                if (any) report(c.status, kEInval);
                return f;
            }
            f.to = blk * a.wb + place * a.wt + l.h * a.wh;
            if (any) {
                f.from = blk * c.sb + place * c.st + l.h * c.sh;
                if constexpr (FMT != kFmt16) f.scale *= __ldg(c.ks + blk * c.ssb + place * c.sst + l.h * c.ssh);
            }
            return f;
        };
        uint4 code[FMT == kFmt16 ? 1 : kIts];
        auto fetch = [&](uint32_t tile) {  // 8 bits: the codes of the tile whose places stand
#pragma unroll
            for (int k = 0; k < kIts; ++k) {
                const int64_t from = s_from[(tile & 1) * kTok + r0 + k * kStep];
                code[k] = in && from >= 0 ? __ldg(reinterpret_cast<const uint4 *>(c.k + from + ch * 16)) : make_uint4(0, 0, 0, 0);
            }
        };
        int g = 0;
        Found now = look(0);
        s_from[i] = now.from;
        named_sync(1, 128);
        if constexpr (FMT != kFmt16) fetch(0);
        // (the four warps meet at every tile: one whose wait gave up goes on with them, and copies nothing)
        for (bool more = true; more; ++key) {  // (l and g stand at the tile, then at the next)
            Found then{-1, -1, 0.0f};
            if (++g == l.halves()) {
                g = 0;
                more = !l.last;
                if (more) l.next(a, sh);
            }
            if (more) then = look(g);
            const uint32_t st = key % S::kKeys, round = key / S::kKeys;
            if (round > 0) {
                if constexpr (LOAD == kGather) {
                    // a warp that has to wait hands over what it has copied first
                    if (!__all_sync(0xffffffffu, bar_test(k_free + 8 * st, (round - 1) & 1))) drain();
                }
                ok = ok && bar_wait(k_free + 8 * st, (round - 1) & 1, dead);
            }
            s_to[st * kTok + i] = now.to;
            s_scale[st * kTok + i] = now.scale;
            const uint32_t into = smem_addr(keys + st * S::kTile);
            if (!ok) {
            } else if constexpr (LOAD == kTma) {
                bar_arrive_warp(k_full + 8 * st);  // (the vectors are another warp's)
            } else if constexpr (LOAD == kGather) {
#pragma unroll
                for (int k = 0; k < kIts; ++k) {
                    const int64_t from = s_from[(key & 1) * kTok + r0 + k * kStep];
                    const bool have = in && from >= 0;
                    copy16(into + swizzled<DP>(r0 + k * kStep, ch), c.k + (have ? from + ch * 16 : 0), have);
                }
                copy_commit();
                if (w1) {
                    copy_wait<2>();
                    shared_to_async();
                    bar_arrive_warp(w1);
                }
                w1 = w0;
                w0 = k_full + 8 * st;
            } else {
#pragma unroll
                for (int k = 0; k < kIts; ++k) {
                    const uint32_t w[4] = {code[k].x, code[k].y, code[k].z, code[k].w};
                    uint32_t v[8];
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        if constexpr (BF16) {
                            v[2 * z] = to_bf16<FMT>(w[z], 0, 1);
                            v[2 * z + 1] = to_bf16<FMT>(w[z], 2, 3);
                        } else {
                            to_half<FMT, false>(w[z], v[2 * z], v[2 * z + 1]);
                        }
                    }
                    const int r = r0 + k * kStep;
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(into + swizzled<DP>(r, 2 * ch)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(into + swizzled<DP>(r, 2 * ch + 1)), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
                }
                shared_to_async();
                bar_arrive_warp(k_full + 8 * st);
            }
            // the next tile's places, for all the warps
            if constexpr (LOAD != kTma) {
                s_from[(key + 1 & 1) * kTok + i] = then.from;
                named_sync(1, 128);
            }
            if constexpr (FMT != kFmt16) {
                if (more) fetch(key + 1);
            }
            now = then;
        }
        drain();
    } else if (LOAD == kTma && warp == 9) {
        // ================= K by the copy engine: lane i is box i of the tile =================
        const int box = in.m.box;
        int g = 0;
        auto look = [&](int &place) {
            const int p = l.base() + g * kTok + lane * box;
            // (what no row sees is not looked up: its block may be gone)
            if (lane * box >= kTok || p >= l.kv || (a.a.window > 0 && p + box - 1 <= l.lo - a.a.window && p >= a.a.sinks)) return -1;
            return (int)block_of(c, a.a.b, l.s, p, place);
        };
        int place = 0, blk = look(place);
        for (bool more = true; more; ++key) {  // (l and g stand at the tile, then at the next)
            const int h = l.h, now = blk, at = place;
            if (++g == l.halves()) {
                g = 0;
                more = !l.last;
                if (more) l.next(a, sh);
            }
            if (more) blk = look(place);
            const uint32_t st = key % S::kKeys, round = key / S::kKeys, boxes = __popc(__ballot_sync(0xffffffffu, now >= 0));
            if (round > 0) ok = bar_wait(k_free + 8 * st, (round - 1) & 1, dead);
            if (!ok) break;
            const uint32_t bar = k_full + 8 * st, into = smem_addr(keys + st * S::kTile) + lane * box * 128;
            if (lane == 0) {
                s_sent_k = key + 1;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(boxes * box * 2 * DP) : "memory");
            }
            __syncwarp();
            if (now >= 0) {
#pragma unroll
                for (int p = 0; p < DP / 64; ++p)
                    asm volatile(
                        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
                            into + p * S::kPanel), "l"(&in.m.k), "r"(bar), "r"(p * 64), "r"(at), "r"(h), "r"(now)
                        : "memory");
            }
        }
    } else if (warp == 11) {
        // ================= queries and their lse to shared memory =================
        // lse of a tile, four rows a lane; asked for a tile ahead
        auto lse_of = [&](int j, float *x) {
            const int row0 = (l.r0 + j) * in.rt, some = min(in.rt, l.rows - row0);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = lane * 4 + k, gr = row0 + r, t = quot(gr, c.div_g);
                x[k] = r < some ? __ldg(a.a.lse + (int64_t)(l.q0 + t) * c.Hq + l.h * c.G + gr - t * c.G) : 0.0f;
            }
        };
        float now[4], then[4];
        lse_of(l.j, now);
        for (int j = l.j;; ++qi) {  // (l and j stand at the tile, then at the next)
            const int row0 = (l.r0 + j) * in.rt, some = min(in.rt, l.rows - row0), q0 = l.q0, h = l.h;
            const bool more = j + 1 < l.end || !l.last;
            if (++j >= l.end && more) {
                l.next(a, sh);
                j = l.j;
            }
            if (more) lse_of(j, then);
            const uint32_t st = qi % S::kRows, round = qi / S::kRows, ls = qi % S::kLess;
            if (qi >= S::kLess) ok = bar_wait(l_free + 8 * ls, (qi / S::kLess - 1) & 1, dead);
            if (!ok) break;
            bool odd = false;
            float less[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // (a row that saw nothing adds nothing, and one with an lse of +inf, as exp(x - inf); neither they nor a column of no row
                // go through the two products, which need not have the same sign)
                const bool none = fabsf(now[k]) == INFINITY;
                odd |= none;
                less[k] = lane * 4 + k >= some || none ? -INFINITY : -fmaf(now[k], a.lse_log2, now[k] * a.lse_log2_rest);
            }
            *reinterpret_cast<float4 *>(s_less + ls * kRowTile + lane * 4) = make_float4(less[0], less[1], less[2], less[3]);
            odd = __any_sync(0xffffffffu, odd);
            if (lane == 0) s_odd[ls] = odd;
            bar_arrive_warp(l_full + 8 * ls);
            if (round > 0) ok = bar_wait(q_free + 8 * st, (round - 1) & 1, dead);
            if (!ok) break;
            const uint32_t into = smem_addr(rows + st * S::kTile);
            if (in.q_map) {
                __syncwarp();
                if (lane == 0) {
                    s_sent = qi + 1;
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(q_full + 8 * st), "r"(in.rt * DP * 2) : "memory");
#pragma unroll
                    for (int p = 0; p < DP / 64; ++p)
                        asm volatile(
                            "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                                into + p * S::kPanel), "l"(&in.q), "r"(q_full + 8 * st), "r"(p * 64), "r"(h * c.G), "r"(q0 + quot(row0, c.div_g))
                            : "memory");
                }
                __syncwarp();
            } else {
                for (int r = lane / (DP / 8); r < (some + 15) / 16 * 16; r += 32 / (DP / 8)) {
                    const int gr = row0 + r, t = quot(gr, c.div_g), qc = lane % (DP / 8);
                    const bool real = r < some && qc * 8 < c.D;
                    const int64_t at = real ? (int64_t)(q0 + t) * a.a.q_t + (int64_t)(h * c.G + gr - t * c.G) * a.a.q_h + qc * 16 : 0;
                    copy16(into + swizzled<DP>(r, qc), a.a.q + at, real);
                }
                copy_commit();
                copy_wait<0>();
                shared_to_async();
                bar_arrive_warp(q_full + 8 * st);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) now[k] = then[k];
            if (!more) break;
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 8) {
        if (*dead) {  // the launch gave up: products and copies that were asked for end before their memory is given back (each wait has a limit)
            if (elect()) commit(ended);
            __syncwarp();
            auto over = [&](uint32_t bar, uint32_t parity) {
                for (uint32_t i = 0; i < kSpin / 64 && !bar_test(bar, parity); ++i) {
                }
            };
            over(ended, 0);
            const uint32_t sent = s_sent;
            for (uint32_t i = sent > S::kRows ? sent - S::kRows : 0; i < sent; ++i) over(q_full + 8 * (i % S::kRows), i / S::kRows & 1);
            const uint32_t sent_k = s_sent_k;
            for (uint32_t i = sent_k > S::kKeys ? sent_k - S::kKeys : 0; i < sent_k; ++i) over(k_full + 8 * (i % S::kKeys), i / S::kKeys & 1);
        }
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
        if (lane == 0 && *dead) report(c.status, kECuda);
    }
    chain_next();
}

using Kernel = void (*)(const ChunkLaunch);
struct Pick {
    Kernel k;
    int smem;
};
template <int FMT, int LOAD>
Pick pick_load(bool bf16, int D) {
    if (D <= 64) return {bf16 ? k_weigh_chunk<true, FMT, 64, LOAD> : k_weigh_chunk<false, FMT, 64, LOAD>, Shape<64>::kSmem};
    return {bf16 ? k_weigh_chunk<true, FMT, 128, LOAD> : k_weigh_chunk<false, FMT, 128, LOAD>, Shape<128>::kSmem};
}
Pick pick(bool bf16, int fmt, int D, bool tma) {
    return fmt == kFmtE4M3 ? pick_load<kFmtE4M3, kConvert>(bf16, D)
         : fmt == kFmtInt8 ? pick_load<kFmtInt8, kConvert>(bf16, D)
         : tma             ? pick_load<kFmt16, kTma>(bf16, D)
                           : pick_load<kFmt16, kGather>(bf16, D);
}

}  // namespace

cudaError_t weigh_init() {
    for (int bf16 = 0; bf16 < 2; ++bf16)
        for (int load = 0; load < 4; ++load)
            for (int D = 64; D <= 128; D += 64) {
                const Pick p = pick(bf16, load == 3 ? (int)kFmt16 : load, D, load == 3);
                const cudaError_t e = cudaFuncSetAttribute(p.k, cudaFuncAttributeMaxDynamicSharedMemorySize, p.smem);
                if (e != cudaSuccess) return e;
            }
    return cudaSuccess;
}

cudaError_t launch_weigh_chunk(const WeighLaunch &a, const CacheMaps &m, bool bf16, int fmt, int sms, cudaStream_t st) {
    const Pick p = pick(bf16, fmt, a.a.c.D, m.box > 0);
    ChunkLaunch l;
    l.w = a;
    l.m = m;
    l.rt = a.a.c.G <= kRowTile ? kRowTile / a.a.c.G * a.a.c.G : kRowTile;
    l.div_rt = fast_div((uint32_t)l.rt);
    l.q_map = encode_rows(a.a, bf16, l.q);
    return launch_chained(p.k, sms, kThreads, p.smem, st, l);
}

}  // namespace lr
