// Attention of many rows over a paged KV cache: chunks of new tokens, and trees of drafted tokens (TREE: a row's mask instead of the
// causal rule, which only the tiles that the drafted tokens or the window's edge lie in are looked at for).
//
// The same one-pass softmax as the step kernel (lr_attend_step.cuh), bound by its two matrix
// products instead of the cache's bytes: 4 D operations a (row, token) pair.  A CTA takes 256 rows
// (tokens x query heads of a KV head) against tiles of 128 cached tokens on the tensor cores of sm_103a (tcgen05):
//   S = Q K^T    both operands in shared memory, 128 x 128 fp32 in tensor memory, one for each half of the rows
//   P = exp2(S)  read, exponentiated, rounded to 16 bits and written over S's upper columns in tensor memory
//   O += P V     P from tensor memory, V from shared memory, O stays in tensor memory
// Sixteen warps: four a half for the softmax, a thread a row; one that issues the products; the others bring
// K, V and Q to shared memory and walk the batch.  The two halves alternate, so that the tensor
// cores work on one while the other's exponentials are taken; a half's weights come in two portions, so that its
// products begin with the first.
//
// O would have to be scaled whenever a row's maximum rises.  The maximum used is instead left behind
// until it is exceeded by 2^kLag, so after the first tiles O hardly ever moves: any reference
// gives the same quotient, and the weights stay at most 2^kLag.
//
// What it takes: a half's chain -- scores, softmax, weights, products -- has to fit while the other half's products
// run, so what is off that chain is kept out of it and out of the loop's code, which 16 warps of six kinds
// share an instruction cache for: hidden scores are set apart (mask_scores: 1,554 -> 1,402 us for 4,096 tokens over
// 32,768, one state repeated as in the next figure), the walk is another warp's (Job), and a warp waits for a barrier with all its lanes
// (a single lane's wait took some 250 cycles even where the phase was over: 2,262 -> 1,596 us).
// Measured (32 query heads on 8 KV heads of 128): 4,096 tokens at the end of 32,768, 16 bits: 1,477 us with inputs in
// turn, 1,396 TFLOP/s, 72% of the library's largest product (on one state again and again 1,353: the card's power differs);
// a half's chain is ~2,700 cycles a tile against 2,048 of products.
#pragma once

#include "lr_attend.cuh"
#include "lr_tensor.cuh"

namespace lr {

namespace {

constexpr int kWeight = 4;  // tiles that a unit's beginning and end take the time of

// How K and V reach shared memory.
enum : int {
    kTma = 0,     // 16-bit cache: the tensor copy engine, one box of tokens of a block at a time
    kGather = 1,  // 16-bit cache of odd blocks: 16 bytes a thread (cp.async)
    kConvert = 2  // 8-bit cache: 16 codes a thread, converted on the way
};

// What the CTA does for one unit, written by the warps that bring its queries: the walk over the batch is
// theirs and the loaders', so that the softmax warps' registers are left to the softmax.
struct Job {
    Unit u;
    int j0, n;          // the CTA's tiles of the unit, from the first
    int whole, last;    // all of the unit's; the CTA's last job
    int c0, c1;         // the CTAs that share the unit
    int slot, slot0;    // where this CTA's and the first one's parts go
};
constexpr int kJobs = 4;
constexpr int kTogether = 6;  // parts that are joined in one step, at most

template <int DP, int FMT, int LOAD, bool TREE>
struct Shape {
    // Warps 0-7 softmax, 8 products.  By the copy engine: 9 K, 10 V, 12-15 queries; else 12-15 K and V, 10
    // and 11 queries.  (12-19 for trees over 8 bits: of few rows, conversion bounds them -- 9,000 cycles a tile of 4 warps, of which
    // the copies' latency is none and a half the other chain --, and the softmax does with fewer registers.)
    static constexpr int kLoaders = LOAD == kConvert && TREE ? 8 : 4, kThreads = 384 + 32 * kLoaders, kLoad = 32 * kLoaders;
    // registers a thread of the softmax warps and of the others: together those of the launch, 512 x 128 or 640 x 96
    static constexpr int kSoftRegs = kLoaders == 8 ? 144 : 192, kOtherRegs = 64;
    static constexpr int kQueryWarp = LOAD == kTma ? 12 : 10, kQueryWarps = LOAD == kTma ? 4 : 2;
    static constexpr int kPanel = kTok * 128;                   // 128 rows of 64 16-bit elements
    static constexpr int kTile = kTok * DP * 2;                 // a tile of K or V, or half of Q, in 16 bits
    static constexpr int kStages = FMT == kFmt16 ? 5 : 4;
    // 8-bit codes on their way: 16 bytes a loading thread and slot, as many as the room takes of the
    // 2 * DP / 16 that a tile of K and one of V make
    static constexpr int kSlots = (DP == 128 ? 14 : 8) * 4 / kLoaders;
    static constexpr int kRaw = FMT == kFmt16 ? 0 : kSlots * kLoad * 16;
    static constexpr int kQ = 2 * kTile;
    static constexpr int kBytes = kQ + kStages * kTile + kRaw;
    static constexpr int kBars = 2 + 2 * kStages + 10 + 4 + 1 + 2 * kJobs + 2;
    static constexpr int kScales = FMT == kFmt16 ? 0 : 4 * 2 * kTok * 4;
    static constexpr int kSmem = kBytes + kScales + 2 * kTok * 8 + kBars * 8 + (kThreads / 32 + 2) * 8 + 29 * 4 + kJobs * sizeof(Job);
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// Tokens that a row does not see have weight zero, but zero times an infinity or a NaN in V is not
// zero.  In a tile that is hidden from some of its rows, such elements of V are therefore set to zero in
// shared memory (clear_row), and the rows that do see them add them at the end (add_lost).  16-bit caches
// only: 8-bit codes are finite, and their scales are kept from hidden weights.
template <bool BF16>
__device__ __forceinline__ const char *v_row(const AttendLaunch &a, const Unit &u, int t) {
    const CacheDev &c = a.c;
    if (t > u.hi || (a.window > 0 && t <= u.lo - a.window && t >= a.sinks)) return nullptr;  // not read: zeros
    int place;
    const int64_t blk = block_of(c, a.b, u.s, t, place);
    return blk < 0 ? nullptr : c.v + blk * c.sb + place * c.st + u.h * c.sh;
}
template <bool BF16>
__device__ __forceinline__ bool lost_in(const uint4 &w) {
    return not_finite<BF16>(w.x) || not_finite<BF16>(w.y) || not_finite<BF16>(w.z) || not_finite<BF16>(w.w);
}
// The elements that are not finite, or all.
template <bool BF16, int DP>
__device__ __noinline__ void clear_row(uint32_t tile, int row, bool all) {
    constexpr uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
    for (int ch = 0; ch < DP / 8; ++ch) {
        const uint32_t at = tile + (ch >> 3) * (kTok * 128) + row * 128 + ((ch ^ row) & 7) * 16;
        uint32_t w[4];
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
        for (int k = 0; k < 4; ++k) {
            if (all || (w[k] & e) == e) w[k] &= 0xffff0000u;
            if (all || (w[k] >> 16 & e) == e) w[k] &= 0xffffu;
        }
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}
template <bool TREE>
__device__ __forceinline__ bool row_sees(const AttendLaunch &a, const Unit &u, int gr, int j) {
    const int t = quot(gr, a.c.div_g);
    if constexpr (TREE) return tree_visible(tree_row(a, u.q0, t, u.ql, u.kv, true), j, a.window, a.sinks);
    return visible(u.kv - u.ql + t, j, a.window, a.sinks);
}
template <bool BF16, bool TREE>
__device__ __noinline__ void add_lost(const AttendLaunch &a, const Unit &u, int tile0, int tile1, int gr, int col, float *o) {
    for (int tile = tile0; tile < tile1; ++tile) {
        const int base = (tile < u.ns ? tile : u.wf + tile - u.ns) * kTok;
        if (!(base + kTok - 1 > u.lo || (a.window > 0 && base <= u.hi - a.window && base + kTok > a.sinks))) continue;
        for (int t = base; t < base + kTok; ++t) {
            if (!row_sees<TREE>(a, u, gr, t)) continue;
            const char *const p = v_row<BF16>(a, u, t);
            for (int d = 0; p && d < 32 && col + d < a.c.D; ++d) {
                const float v = unpack16<BF16>(*reinterpret_cast<const uint16_t *>(p + (col + d) * 2)).x;
                if (!(fabsf(v) < INFINITY)) o[d] += v;
            }
        }
    }
}

// V's scales over 8-bit codes in fp16: code * (2^e * rest) with 1 <= |rest| < 2.  The power of two goes to the codes as
// they are converted, the rest to the weights, which so are as far from the ends of fp16's range as those of a 16-bit
// cache, however large or small V is.  The codes get 2^(e + 1), and the sums are halved: a product below 2^-14 that fp16 rounds
// by up to 2^-25 is off by half that times the rest, less than 2^-25 of V.  e + 1 stays in [-24, 5], where the
// products are finite; what a scale has beyond is in the rest: weights of up to 2^4 stay numbers with
// scales of up to 2^15.
constexpr int kLeast = -24, kMost = 5;
__device__ __forceinline__ int power(float scale) { return min(max((int)(__float_as_uint(scale) >> 23 & 0xff) - 126, kLeast), kMost); }
__device__ __forceinline__ float rest_of(float scale) { return scale * __uint_as_float((uint32_t)(128 - power(scale)) << 23); }
// The codes' power of two as fp16's bits; of e4m3 2^8 as much, for the codes that to_half_times makes.
template <int FMT>
__device__ __forceinline__ uint32_t power_of(float scale) {
    return __half_as_ushort(__float2half_rn(__uint_as_float((uint32_t)(127 + power(scale) + (FMT == kFmtE4M3 ? 8 : 0)) << 23)));
}
template <int FMT>
__device__ __forceinline__ uint32_t half_times(uint32_t two) {
    uint32_t r = 0;
    if constexpr (FMT == kFmtInt8) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(two), "r"(0xe480e480u));  // -1152 times it
    return r;
}
// Four codes (0, 1), (2, 3) times `two`.  int8: (1024 + (code + 128)) * two - 1152 * two in one rounding.  e4m3:
// the code's bits moved to fp16's places are 2^-8 times its value (and its NaN a number, which hidden weights need).
template <int FMT>
__device__ __forceinline__ void to_half_times(uint32_t w, uint32_t two, uint32_t shift, uint32_t &a, uint32_t &b) {
    if constexpr (FMT == kFmtE4M3) {
        a = __byte_perm(w, 0, 0x1404);
        b = __byte_perm(w, 0, 0x3424);
        a = (a & 0x80008000u) | ((a >> 1) & 0x3f803f80u);
        b = (b & 0x80008000u) | ((b >> 1) & 0x3f803f80u);
        asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(a) : "r"(two));
        asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(b) : "r"(two));
    } else {
        w ^= 0x80808080u;
        a = __byte_perm(w, 0x64646464u, 0x4140);
        b = __byte_perm(w, 0x64646464u, 0x4342);
        asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(a) : "r"(two), "r"(shift));
        asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(b) : "r"(two), "r"(shift));
    }
}

struct ChunkLaunch {
    AttendLaunch a;
    CacheMaps m;
    CUtensorMap q;   // boxes of 64 elements of 128 rows: the query heads of a KV head, times tokens
    int32_t q_map;   // there is one: their number divides 128
};

// Scores that a row does not see to -inf (at most `last`, and above `low` or below `sink` it does), in tensor
// memory and out of the way of the loop, which nearly every tile goes through without; kbad: a bit for each
// token whose block is out of range or whose K has a scale that is not finite, to NaN where a row sees it.
__device__ __noinline__ void mask_scores(uint32_t ts, int last, int low, int sink, const uint32_t *kbad) {
    auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };
#pragma unroll 1
    for (int k0 = 0; k0 < kTok; k0 += 32) {
        const uint32_t see = below(last + 1 - k0) & (~below(low + 1 - k0) | below(sink - k0)), nan = kbad ? kbad[k0 / 32] : 0u;
        if (__all_sync(0xffffffffu, see == ~0u && nan == 0u)) continue;
        float s[32];
        tm_load(s, ts + k0);
        tm_load_wait(s);
        if (nan) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (nan >> k & 1) s[k] = __uint_as_float(0x7fffffffu);
        }
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (!(see >> k & 1)) s[k] = -INFINITY;
        tm_store(ts + k0, reinterpret_cast<uint32_t *>(s));
        tm_store(ts + k0 + 16, reinterpret_cast<uint32_t *>(s) + 16);
    }
    tm_store_wait();
}
// Records a block out of range among those of sequence s's tokens j + k, k a bit of `seen` (the others have a scale that is not
// finite).
__device__ __noinline__ void report_blocks(const AttendLaunch &a, int s, int j, uint32_t seen) {
    int place;
    for (; seen; seen &= seen - 1)
        if (block_of(a.c, a.b, s, j + __ffs(seen) - 1, place) < 0) {
            report(a.c.status, kEInval);
            break;
        }
    __syncwarp();
}
// The same for the rows of a tree, whose context and drafted tokens are hidden by different rules.  A block out of range is
// recorded here, where a row sees it: what is looked up is what a row can see that names nothing.
__device__ __noinline__ void mask_tree(uint32_t ts, const AttendLaunch &a, int s, int q0, int t, int ql, int kv, int at, int base,
                                       const uint32_t *kbad) {
    const TreeRow row = tree_row_at(a, q0, t, ql, kv, at);
#pragma unroll 1
    for (int k0 = 0; k0 < kTok; k0 += 32) {
        const uint32_t see = tree_sees(row, base + k0, a.window, a.sinks), nan = kbad ? kbad[k0 / 32] : 0u;
        if (__all_sync(0xffffffffu, see == ~0u && nan == 0u)) continue;
        if (nan) report_blocks(a, s, base + k0, see & nan);
        float x[32];
        tm_load(x, ts + k0);
        tm_load_wait(x);
        if (nan) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (nan >> k & 1) x[k] = __uint_as_float(0x7fffffffu);
        }
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (!(see >> k & 1)) x[k] = -INFINITY;
        tm_store(ts + k0, reinterpret_cast<uint32_t *>(x));
        tm_store(ts + k0 + 16, reinterpret_cast<uint32_t *>(x) + 16);
    }
    tm_store_wait();
}
// Whether a row sees a token whose V has a scale that is not finite (its weights were multiplied by zero).
template <bool TREE>
__device__ __noinline__ bool sees_lost(const AttendLaunch &a, const Unit &u, int tile0, int tile1, int gr) {
    const CacheDev &c = a.c;
    for (int tile = tile0; tile < tile1; ++tile) {
        const int base = (tile < u.ns ? tile : u.wf + tile - u.ns) * kTok;
        for (int t = base; t < base + kTok; ++t) {
            if (!row_sees<TREE>(a, u, gr, t)) continue;
            int place;
            const int64_t blk = block_of(c, a.b, u.s, t, place);
            if (blk >= 0 && !(fabsf(c.vs[blk * c.ssb + place * c.sst + u.h * c.ssh]) < INFINITY)) return true;
        }
    }
    return false;
}

// Joins the parts of 32 rows of a unit, in the order of the CTAs: a lane first a row's maximum and sum, then four
// elements each of 16 rows at a time (of 2 x 8 with 64 elements), their loads in flight together.
// The parts are those of CTA c0 + k * step.  LAST: to the outputs; else to the first part's own place, as a part of others.
template <bool BF16, int DP, bool LAST>
__device__ __noinline__ void join_rows(const AttendLaunch &a, const Unit &u, int c0, int parts, int slot0, int row0, int step) {
    constexpr int kLanes = DP / 4, kTwo = 32 / kLanes, kStep = 16;
    const CacheDev &c = a.c;
    const int lane = threadIdx.x % 32, sub = lane / kLanes, e = lane % kLanes * 4;
    auto at = [&](int k, int r) { return (int64_t)(k == 0 ? slot0 : 2 * (c0 + k * step)) * 256 + r; };
    const bool mine = row0 + lane < u.rows;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) mm = fmaxf(mm, mine ? __ldcg(&a.part_ml[at(k, row0 + lane)].x) : 0.0f);
    for (int r0 = row0; r0 < min(u.rows, row0 + 32); r0 += kStep) {
        float4 acc[kStep / kTwo];
#pragma unroll
        for (int z = 0; z < kStep / kTwo; ++z) acc[z] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        ll = 0.0f;
        for (int k = 0; k < parts; ++k) {
            float4 w[kStep / kTwo];
            const float4 *const from = reinterpret_cast<const float4 *>(a.part_o + at(k, r0 + sub) * 128 + e);
#pragma unroll
            for (int z = 0; z < kStep / kTwo; ++z) {  // (asked for together, whether they count or not)
                w[z] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (r0 + z * kTwo + sub < u.rows)
                    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(w[z].x), "=f"(w[z].y), "=f"(w[z].z), "=f"(w[z].w) : "l"(from + z * kTwo * 32));
            }
            const float2 ml = mine ? __ldcg(a.part_ml + at(k, row0 + lane)) : make_float2(-INFINITY, 0.0f);
            const float f = ml.x == -INFINITY ? 0.0f : exp2_fast(ml.x - mm);  // (one that saw nothing: no part of it)
            ll += ml.y == 0.0f ? 0.0f : ml.x == -INFINITY ? ml.y : ml.y * f;
#pragma unroll
            for (int z = 0; z < kStep / kTwo; ++z) {
                const float g = __shfl_sync(0xffffffffu, f, r0 - row0 + z * kTwo + sub);
                const bool on = g != 0.0f;
                acc[z].x += on ? w[z].x * g : 0.0f;
                acc[z].y += on ? w[z].y * g : 0.0f;
                acc[z].z += on ? w[z].z * g : 0.0f;
                acc[z].w += on ? w[z].w * g : 0.0f;
            }
        }
#pragma unroll
        for (int z = 0; z < kStep / kTwo; ++z) {
            const int r = r0 + z * kTwo + sub;
            const float l = __shfl_sync(0xffffffffu, ll, r - row0);
            const int gr = u.qt * 256 + r, t = quot(gr, c.div_g), hd = u.h * c.G + gr - t * c.G;
            const float iv = l == 0.0f ? 0.0f : 1.0f / l;
            if (!LAST && r < u.rows)
                *reinterpret_cast<float4 *>(a.part_o + at(0, r) * 128 + e) = acc[z];
            if (LAST && r < u.rows && e < c.D)
                *reinterpret_cast<uint2 *>(a.out + (int64_t)(u.q0 + t) * a.o_t + (int64_t)hd * a.o_h + e * 2) =
                    make_uint2(pack16<BF16>(acc[z].x * iv, acc[z].y * iv), pack16<BF16>(acc[z].z * iv, acc[z].w * iv));
        }
    }
    if constexpr (!LAST) {
        if (mine) a.part_ml[at(0, row0 + lane)] = make_float2(mm, ll);
        return;
    }
    if (a.lse && mine) {
        const int gr = u.qt * 256 + row0 + lane, t = quot(gr, c.div_g), hd = u.h * c.G + gr - t * c.G;
        a.lse[(int64_t)(u.q0 + t) * c.Hq + hd] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
    }
}

template <bool BF16, int FMT, int DP, int LOAD, bool TREE>
__global__ void __launch_bounds__(Shape<DP, FMT, LOAD, TREE>::kThreads, 1) k_attend_chunk(const __grid_constant__ ChunkLaunch in) {
    using S = Shape<DP, FMT, LOAD, TREE>;
    const AttendLaunch &a = in.a;
    constexpr int kThreads = S::kThreads, kLoad = S::kLoad;
    constexpr int kKvArrive = LOAD == kTma ? 1 : S::kLoaders;  // arrivals that hand over a tile: one a warp
    constexpr int kStages = S::kStages;
    constexpr float kLag = BF16 || FMT == kFmt16 ? 8.0f : 4.0f;
    constexpr bool kSplit = FMT != kFmt16 && !BF16;  // V's scales are split (below)
    // (no static shared memory, so that the tiles start where the swizzle's 1,024-byte pattern does)
    extern __shared__ __align__(1024) char smem[];
    char *const tiles = smem + S::kQ;
    char *const raw = tiles + kStages * S::kTile;
    float *const scales = reinterpret_cast<float *>(smem + S::kBytes);                                    // [4][K, V][token]
    int64_t *const places = reinterpret_cast<int64_t *>(smem + S::kBytes + S::kScales);                   // [2][token]
    uint64_t *const bars = reinterpret_cast<uint64_t *>(places + 2 * kTok);
    long long *const scratch = reinterpret_cast<long long *>(bars + S::kBars);
    Job *const jobs = reinterpret_cast<Job *>(scratch + kThreads / 32 + 2);
    int *const s_bad = reinterpret_cast<int *>(jobs + kJobs);  // [4] of a tile, 1: s_kbad names tokens, 2: a scale of V is not finite
    int *const s_lost = s_bad + 4;                             // [half][2] the last scan that found V not finite
    int &s_dead = s_bad[8];
    uint32_t &s_tmem = *reinterpret_cast<uint32_t *>(s_bad + 9);
    uint32_t *const s_kbad = reinterpret_cast<uint32_t *>(s_bad + 10);  // [4][4] a bit a token: its scores are NaN
    uint32_t *const s_sent = s_kbad + 16;  // tiles of K and of V, and units of Q, that the copy engine was asked for
    const uint32_t b0 = smem_addr(bars);
    const uint32_t q_full = b0, q_free = b0 + 8, kv_full = b0 + 16, kv_free = kv_full + 8 * kStages, s_full = kv_free + 8 * kStages,
                   p_half = s_full + 16, p_full = p_half + 16, o_full = p_full + 16, o_free = o_full + 16, sc_full = o_free + 16,
                   ended = sc_full + 32, job_full = ended + 8, job_free = job_full + 8 * kJobs, scanned = job_free + 8 * kJobs;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const CacheDev &c = a.c;

    chain_wait();
    Cursor<256, kTok, kWeight> cu;
    Share sh;
    if (!take_share<256, kTok, kWeight, kThreads, 4>(a, cu, sh, scratch)) {
        chain_next();
        return;
    }
    if (tid == 0) {
        bar_init(q_full, S::kQueryWarps);
        bar_init(q_free, 1);
        for (int i = 0; i < kStages; ++i) {
            bar_init(kv_full + 8 * i, kKvArrive);
            bar_init(kv_free + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(s_full + 8 * i, 1);
            bar_init(p_full + 8 * i, 4);
            bar_init(p_half + 8 * i, 4);
            bar_init(o_full + 8 * i, 1);
            bar_init(o_free + 8 * i, 4);
        }
        for (int i = 0; i < 4; ++i) bar_init(sc_full + 8 * i, kKvArrive);
        bar_init(ended, 1);
        for (int i = 0; i < kJobs; ++i) {
            bar_init(job_full + 8 * i, 1);
            bar_init(job_free + 8 * i, 8);
        }
        bar_init(scanned, 4);
        bar_init(scanned + 8, 4);
        for (int i = 0; i < 4; ++i) s_lost[i] = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
        s_dead = 0;
        s_sent[0] = s_sent[1] = s_sent[2] = 0;
    }
    if (warp == 8) {
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
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftRegs));
        const int half = warp / 4, r = tid;  // row of the unit
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tm + half * 128 + lanes, to = tm + 256 + half * 128 + lanes;
        uint32_t n_s = 0, n_o = 0, n_scan = 0;
        int x = 0;  // the CTA's tile
        bool ok = true;
        for (int frag = 0;; ++frag) {
            const Job &job = jobs[frag % kJobs];
            const Unit &u = job.u;
            ok = bar_wait(job_full + 8 * (frag % kJobs), frag / kJobs & 1, dead);
            if (!ok) break;
            const int n = job.n;
            const bool last_job = job.last;
            if (half == 1 && u.rows <= 128) {
                x += n;
                bar_arrive_warp(job_free + 8 * (frag % kJobs));
                if (last_job) break;
                continue;
            }
            const int gr = u.qt * 256 + r, t = quot(gr, c.div_g);
            const bool real = r < u.rows;
            const int pos = TREE ? tree_row(a, u.q0, t, u.ql, u.kv, real).at : real ? u.kv - u.ql + t : -1;
            // positions of the half's first and last row
            const int f0 = u.qt * 256 + half * 128, f1 = u.qt * 256 + min(u.rows, half * 128 + 128) - 1;
            const int lo = TREE ? u.lo : u.kv - u.ql + quot(f0, c.div_g), hi = TREE ? u.hi : u.kv - u.ql + quot(f1, c.div_g);
            float mref = -INFINITY;  // the maximum that the weights refer to, times scale * log2(e)
            float2 l2 = make_float2(0.0f, 0.0f);
            bool lost = false;  // values of V that were set to zero
            const int ulo = u.lo, uhi = u.hi, ns = u.ns, skip = u.wf - u.ns;
            for (int j = 0, tile = job.j0; j < n; ++j, ++tile, ++x) {
                const int base = (tile < ns ? tile : tile + skip) * kTok;
                const int slot = x & 3;
                const bool masked = base + kTok - 1 > lo || (a.window > 0 && base <= hi - a.window && base + kTok > a.sinks);
                [[maybe_unused]] bool wipe = false, gone = false, clear = false;
                if constexpr (FMT == kFmt16) {
                    // (hidden from a row of either half: they share V)
                    if (base + kTok - 1 > ulo || (a.window > 0 && base <= uhi - a.window && base + kTok > a.sinks)) {
                        // a thread a token: is all of its V finite?
                        bool bad = false;
                        const char *const p = v_row<BF16>(a, u, base + (tid & 127));
                        for (int d = 0; p && d < c.D; d += 8) bad |= lost_in<BF16>(__ldg(reinterpret_cast<const uint4 *>(p + d * 2)));
                        gone = LOAD == kTma && !p;  // no token of the unit: whatever was copied, or nothing
                        int *const found = s_lost + half * 2 + (n_scan & 1);
                        if (bad) *found = x;
                        bar_arrive_warp(scanned + 8 * half);
                        ok = bar_wait(scanned + 8 * half, n_scan & 1, dead);
                        if (!ok) break;
                        ++n_scan;
                        lost |= *reinterpret_cast<volatile int *>(found) == x;
                        wipe = bad || gone;
                        clear = __any_sync(0xffffffffu, wipe);
                    }
                }
                // (the scores before the scales and before V: a half that skips units may be ahead of those barriers by
                // phases, which their parity does not tell apart; this tile's scores mean that K has landed, and all before it)
                ok = bar_wait(s_full + 8 * half, n_s & 1, dead) && (FMT == kFmt16 || bar_wait(sc_full + 8 * slot, x >> 2 & 1, dead));
                if (!ok) break;
                if constexpr (FMT == kFmt16) {
                    if (clear) {
                        const uint32_t v = 2 * x + 1;
                        ok = bar_wait(kv_full + 8 * (v % kStages), v / kStages & 1, dead);
                        if (!ok) break;
                        if (wipe) clear_row<BF16, DP>(smem_addr(tiles + v % kStages * S::kTile), tid & 127, gone);
                        shared_to_async();
                        __syncwarp();
                    }
                }
                ++n_s;
                const float *const ks = scales + slot * 2 * kTok, *const vs = ks + kTok;
                after_sync();
                const int flags = *const_cast<volatile int *>(s_bad + slot);
                if (TREE && (masked || (flags & 1)))
                    mask_tree(ts, a, u.s, u.q0, t, u.ql, u.kv, pos, base, flags & 1 ? s_kbad + slot * 4 : nullptr);
                else if (masked || (flags & 1))
                    mask_scores(ts, pos - base, a.window > 0 ? pos - a.window - base : -1, a.sinks - base,
                                flags & 1 ? s_kbad + slot * 4 : nullptr);
                // 32 scores from tensor memory as they enter the softmax: times the scales of K
                auto enter = [&](float *s, int k0) {
                    if constexpr (FMT != kFmt16) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 f = *reinterpret_cast<const float4 *>(ks + k0 + k);
                            const float2 e = mul2(make_float2(s[k], s[k + 1]), make_float2(f.x, f.y)), g = mul2(make_float2(s[k + 2], s[k + 3]), make_float2(f.z, f.w));
                            s[k] = e.x;
                            s[k + 1] = e.y;
                            s[k + 2] = g.x;
                            s[k + 3] = g.y;
                        }
                    }
                };
                // The first 64 scores are read again for their weights: 128 would not fit the registers.
                float sa[32], sb[64];
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto most = [&](const float *s) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
#pragma unroll
                        for (int z = 0; z < 4; ++z) mx[z] = fmaxf(fmaxf(mx[z], s[k + z]), s[k + 4 + z]);
                };
                tm_load(sb, ts);
                tm_load(sb + 32, ts + 32);
                tm_load_wait(sb);
                tm_load_wait(sb + 32);
                enter(sb, 0);
                most(sb);
                enter(sb + 32, 32);
                most(sb + 32);
                tm_load(sb, ts + 64);
                tm_load(sb + 32, ts + 96);
                tm_load_wait(sb);
                tm_load_wait(sb + 32);
                enter(sb, 64);
                most(sb);
                enter(sb + 32, 96);
                most(sb + 32);
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
                            tm_load(sa, to + k);
                            tm_load_wait(sa);
#pragma unroll
                            for (int z = 0; z < 32; ++z) sa[z] *= f;
                            tm_store(to + k, reinterpret_cast<uint32_t *>(sa));
                            tm_store(to + k + 16, reinterpret_cast<uint32_t *>(sa) + 16);
                        }
                    }
                }
                const float neg = mref == -INFINITY ? 0.0f : -mref;
                const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), neg2 = make_float2(neg, neg);
                // the weights of 32 tokens, to the upper half of the scores' columns
                auto weigh = [&](const float *s, int k0) {
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        float2 e = fma2(make_float2(s[k], s[k + 1]), sc2, neg2), g = fma2(make_float2(s[k + 2], s[k + 3]), sc2, neg2);
                        e.x = exp2_fast(e.x);
                        e.y = exp2_fast(e.y);
                        g.x = exp2_fast(g.x);
                        g.y = exp2_fast(g.y);
                        l2 = add2(l2, add2(e, g));
                        if constexpr (FMT != kFmt16) {
                            const float4 f = *reinterpret_cast<const float4 *>(vs + k0 + k);
                            e = mul2(e, make_float2(f.x, f.y));
                            g = mul2(g, make_float2(f.z, f.w));
                        }
                        p[k / 2] = pack16<BF16>(e.x, e.y);
                        p[k / 2 + 1] = pack16<BF16>(g.x, g.y);
                    }
                    tm_store(ts + 64 + k0 / 2, p);
                };
                tm_load(sa, ts);
                weigh(sb, 64);
                weigh(sb + 32, 96);
                tm_store_wait();
                before_sync();
                bar_arrive_warp(p_half + 8 * half);  // the products of these may begin
                tm_load_wait(sa);
                tm_load(sb, ts + 32);
                enter(sa, 0);
                weigh(sa, 0);
                tm_load_wait(sb);
                enter(sb, 32);
                weigh(sb, 32);
                tm_store_wait();
                if (FMT != kFmt16 && (flags & 2)) lost = true;
                before_sync();
                bar_arrive_warp(p_full + 8 * half);
            }
            // ---- the unit ends here, for this CTA ----
            ok = ok && bar_wait(o_full + 8 * half, n_o & 1, dead);
            if (!ok) break;
            ++n_o;
            after_sync();
            const float l = l2.x + l2.y;
            const bool whole = job.whole;
            const int hd = u.h * c.G + gr - t * c.G;
            const int64_t slot = job.slot;
            char *const po = a.out + (int64_t)(u.q0 + t) * a.o_t + (int64_t)hd * a.o_h;
            float *const pw = a.part_o + (slot * 256 + r) * 128;
            constexpr float kHalf = kSplit ? 0.5f : 1.0f;  // (V's codes were taken twice)
            const float inv = l == 0.0f ? 0.0f : kHalf / l;
            bool gone = false;
#pragma unroll 1
            for (int k = 0; k < DP; k += 32) {  // (short code: it is fetched anew for each unit)
                float o[32];
                __syncwarp();
                tm_load(o, to + k);
                tm_load_wait(o);
                if constexpr (FMT == kFmt16) {
                    if (lost && real) {
                        float y[32];
#pragma unroll
                        for (int z = 0; z < 32; ++z) y[z] = o[z];
                        add_lost<BF16, TREE>(a, u, job.j0, job.j0 + n, gr, k, y);
#pragma unroll
                        for (int z = 0; z < 32; ++z) o[z] = y[z];
                    }
                }
                if constexpr (FMT != kFmt16) {
                    if (lost && real && (k > 0 ? gone : (gone = sees_lost<TREE>(a, u, job.j0, job.j0 + n, gr)))) {
#pragma unroll
                        for (int z = 0; z < 32; ++z) o[z] = __uint_as_float(0x7fffffffu);
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
                    for (int z = 0; z < 32; z += 4) *reinterpret_cast<float4 *>(pw + k + z) = make_float4(o[z] * kHalf, o[z + 1] * kHalf, o[z + 2] * kHalf, o[z + 3] * kHalf);
                }
            }
            __syncwarp();
            before_sync();
            bar_arrive_warp(o_free + 8 * half);
            if (real) {
                if (!whole) a.part_ml[slot * 256 + r] = make_float2(mref, l);
                else if (a.lse) a.lse[(int64_t)(u.q0 + t) * c.Hq + hd] = l == 0.0f ? -INFINITY : (mref + log2f(l)) * 0.69314718f;
            }
            if (!whole) {
                // The warps that have the same rows of the unit, one a CTA: the last of them joins the parts, in the
                // order of the CTAs whichever came last.
                const int c0 = job.c0, c1 = job.c1;
                const int parts = c1 - c0 + 1;
                // whether this warp is the last of `all` to come to counter n, which then starts again
                auto last_of = [&](int n, int all) {
                    uint32_t before = 0;
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) {
                        before = atomicAdd(a.done + n * 8 + warp, 1u);
                        if (before == (uint32_t)(all - 1)) a.done[n * 8 + warp] = 0;
                    }
                    before = __shfl_sync(0xffffffffu, before, 0);
                    __threadfence();
                    return before == (uint32_t)(all - 1);
                };
                if (TREE && parts > kTogether) {
                    // Many parts in two steps, so that as many SMs take part as there are groups (19 parts of a context of 200,001
                    // tokens, joined by one warp a row's 32: 75 us of 218).  Groups have counters of their own, at their first CTA.
                    const int group = parts > 36 ? 12 : parts > 16 ? 6 : 4, g = ((int)blockIdx.x - c0) / group, first = g * group;
                    const int n = min(group, parts - first), groups = (parts + group - 1) / group;
                    if (last_of(g == 0 ? c0 : (int)gridDim.x + c0 + first, n)) {
                        join_rows<BF16, DP, false>(a, u, c0 + first, n, g == 0 ? job.slot0 : 2 * (c0 + first), warp * 32, 1);
                        if (last_of(2 * (int)gridDim.x + c0, groups)) join_rows<BF16, DP, true>(a, u, c0, groups, job.slot0, warp * 32, group);
                    }
                } else if (last_of(c0, parts)) {
                    join_rows<BF16, DP, true>(a, u, c0, parts, job.slot0, warp * 32, 1);
                }
            }
            bar_arrive_warp(job_free + 8 * (frag % kJobs));
            if (last_job) break;
        }
    } else if (LOAD != kTma && warp >= 12) {
        // ================= K and V to shared memory, by threads =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOtherRegs));
        const int i = tid - 384;
        uint32_t item = 0;
        bool ok = true;
        // 16-bit copies complete in order: the barriers of the last two groups wait for theirs
        uint32_t w0 = 0, w1 = 0;
        auto landed = [&](uint32_t bar) {
            copy_commit();
            if (w1) {
                copy_wait<2>();
                shared_to_async();
                bar_arrive_warp(w1);
            }
            w1 = w0;
            w0 = bar;
        };
        auto drain = [&]() {
            copy_wait<0>();
            shared_to_async();
            if (w1) bar_arrive_warp(w1);
            if (w0) bar_arrive_warp(w0);
            w0 = w1 = 0;
        };
        // where token i of the tile at cursor p is, with its scales
        struct Found {
            int64_t off;
            float ks, vs;
            bool bad;
        };
        auto look = [&](const Cursor<256, kTok, kWeight> &p) {
            Found f{-1, 1.0f, 0.0f, false};
            const int t = p.base() + i;
            if (i >= kTok || t > p.u.hi || (a.window > 0 && t <= p.u.lo - a.window && t >= a.sinks)) return f;
            int place;
            const int64_t blk = block_of(c, a.b, p.u.s, t, place);
            if (blk < 0) {
                f.bad = true;
                if constexpr (!TREE) report(c.status, kEInval);  // (mask_tree does)
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
        constexpr int CH = FMT == kFmt16 ? DP / 8 : DP / 16, kStep = kLoad / CH, kIts = kTok / kStep;
        // (8 bits: eight neighbouring threads write two rows' 64 elements, which lie in different banks; eight pieces of one row would not)
        constexpr bool kTwoRows = FMT != kFmt16 && CH == 8;
        const int ch = kTwoRows ? (i & 3) | (i >> 1 & 4) : i % CH, r0 = kTwoRows ? (i >> 2 & 1) | i >> 4 << 1 : i / CH;
        const bool in = ch * (FMT == kFmt16 ? 8 : 16) < c.D;
        auto put = [&](int x, const Found &f) {
            if (i >= kTok) return;
            if constexpr (kSplit) places[(x & 1) * kTok + i] = (int64_t)((uint64_t)power_of<FMT>(f.vs) << 48 | ((uint64_t)f.off << 16 >> 16));
            else places[(x & 1) * kTok + i] = f.off;
            // blocks out of range and scales that are not finite are kept from rows that do not see them
            bool kb = f.bad;
            int flags = 0;
            if constexpr (FMT != kFmt16) {
                kb |= !(fabsf(f.ks) < INFINITY);
                const bool vb = !(fabsf(f.vs) < INFINITY);
                scales[(x & 3) * 2 * kTok + i] = kb ? 1.0f : f.ks;
                scales[(x & 3) * 2 * kTok + kTok + i] = vb ? 0.0f : kSplit ? rest_of(f.vs) : f.vs;
                flags |= __any_sync(0xffffffffu, vb) ? 2 : 0;
            }
            const unsigned kw = __ballot_sync(0xffffffffu, kb);
            flags |= kw ? 1 : 0;
            if (lane == 0) s_kbad[(x & 3) * 4 + warp - 12] = kw;
            if (lane == 0 && flags) atomicOr(s_bad + (x & 3), flags);
        };
        // stage of the next item, free to be written
        auto stage = [&]() {
            const uint32_t st = item % kStages, round = item / kStages;
            if (round > 0) {
                if constexpr (FMT == kFmt16) {
                    // a warp that has to wait hands over what it has copied first
                    if (!__all_sync(0xffffffffu, bar_test(kv_free + 8 * st, (round - 1) & 1))) drain();
                }
                ok = ok && bar_wait(kv_free + 8 * st, (round - 1) & 1, dead);
            }
            return st;
        };
        // 8-bit codes: copy number n of this thread (kIts an item, K and V in turn) of the tile in places slot `at`
        uint32_t ahead = 0;  // copies requested
        auto request = [&](bool any) {
            const uint32_t it = ahead / kIts, k = ahead % kIts;
            if (any) {
                int64_t off = places[(it >> 1 & 1) * kTok + r0 + k * kStep];
                if constexpr (kSplit) off = (int64_t)((uint64_t)off << 16) >> 16;
                const bool have = in && off >= 0;
                copy16(smem_addr(raw + (ahead % S::kSlots * kLoad + i) * 16), (it & 1 ? c.v : c.k) + (have ? off + ch * 16 : 0), have);
            }
            copy_commit();
            ++ahead;
        };
        if (i < 4) s_bad[i] = 0;
        named_sync(1, kLoad);
        put(0, look(cu));
        named_sync(1, kLoad);
        if constexpr (FMT != kFmt16) {
            static_assert(FMT == kFmt16 || S::kSlots <= 2 * kIts, "the first requests are the first tile's");
            for (int k = 0; k < S::kSlots; ++k) request(true);
        }
        for (int x = 0, more = 1; more; ++x) {  // (cu stands at tile x, then at x + 1)
            bar_arrive_warp(sc_full + 8 * (x & 3));  // the tile's scales and flag
            more = cu.more();
            Found f{-1, 1.0f, 0.0f, false};
            if (more) {
                cu.next(a, sh);
                f = look(cu);
            }
            if constexpr (FMT == kFmt16) {
                for (int y = 0; y < 2; ++y, ++item) {
                    const uint32_t st = stage();
                    const uint32_t to = smem_addr(tiles + st * S::kTile);
                    const char *const from = y ? c.v : c.k;
#pragma unroll
                    for (int k0 = 0; k0 < kIts; k0 += 8) {
                        int64_t off[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) off[k] = places[(x & 1) * kTok + r0 + (k0 + k) * kStep];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const bool have = in && off[k] >= 0;
                            copy16(to + swizzled<DP>(r0 + (k0 + k) * kStep, ch), from + (have ? off[k] + ch * 16 : 0), have);
                        }
                    }
                    landed(kv_full + 8 * st);
                }
            }
            // the next tile's places (8-bit: before this tile's codes are taken, in whose room its own are requested)
            if (i == 0) s_bad[(x + 1) & 3] = 0;
            named_sync(1, kLoad);
            if (more) put(x + 1, f);
            named_sync(1, kLoad);
            if constexpr (FMT != kFmt16) {
                for (int y = 0; y < 2; ++y, ++item) {
                    const uint32_t st = stage();
                    const uint32_t to = smem_addr(tiles + st * S::kTile);
                    // four pieces (or what there are) at a time: read, converted and written, then their slots requested again
                    constexpr int kFour = kIts < 4 ? kIts : 4;
                    for (int k0 = 0; k0 < kIts; k0 += kFour) {
                        uint32_t w[kFour][4];
                        copy_wait<S::kSlots - kFour>();
#pragma unroll
                        for (int k = 0; k < kFour; ++k)
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                         : "=r"(w[k][0]), "=r"(w[k][1]), "=r"(w[k][2]), "=r"(w[k][3])
                                         : "r"(smem_addr(raw + ((item * kIts + k0 + k) % S::kSlots * kLoad + i) * 16)) : "memory");
#pragma unroll
                        for (int k = 0; k < kFour; ++k) {
                            const int r = r0 + (k0 + k) * kStep;
                            uint32_t v[8];
                            if constexpr (BF16) {
#pragma unroll
                                for (int z = 0; z < 4; ++z) {
                                    v[2 * z] = to_bf16<FMT>(w[k][z], 0, 1);
                                    v[2 * z + 1] = to_bf16<FMT>(w[k][z], 2, 3);
                                }
                            } else if (y) {
                                const uint32_t two = __byte_perm(reinterpret_cast<const uint32_t *>(places + (x & 1) * kTok + r)[1], 0, 0x3232);
                                const uint32_t shift = half_times<FMT>(two);
#pragma unroll
                                for (int z = 0; z < 4; ++z) to_half_times<FMT>(w[k][z], two, shift, v[2 * z], v[2 * z + 1]);
                            } else {
#pragma unroll
                                for (int z = 0; z < 4; ++z) to_half<FMT, false>(w[k][z], v[2 * z], v[2 * z + 1]);
                            }
                            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + swizzled<DP>(r, 2 * ch)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + swizzled<DP>(r, 2 * ch + 1)), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
                        }
                        // the copies that take these slots next are of this tile's V or of the next tile
#pragma unroll
                        for (int k = 0; k < kFour; ++k) request(ahead / (2 * kIts) <= (uint32_t)x + (more ? 1 : 0));
                    }
                    shared_to_async();
                    bar_arrive_warp(kv_full + 8 * st);
                }
            }
        }
        if constexpr (FMT == kFmt16) drain();
        copy_wait<0>();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOtherRegs));
        if (LOAD == kTma && (warp == 9 || warp == 10)) {
            // ================= K and V to shared memory, by the copy engine =================
            // lane i: box i of the tile; warp 9 takes K, warp 10 V
            const int box = in.m.box;
            const bool is_v = warp == 10;
            const CUtensorMap *const map = is_v ? &in.m.v : &in.m.k;
            uint32_t item = is_v, sent = 0;
            bool ok = true;
            auto look = [&](int &place, bool &bad) {
                const int t = cu.base() + lane * box;
                bad = false;
                if (lane * box >= kTok || t > cu.u.hi || (a.window > 0 && t + box - 1 <= cu.u.lo - a.window && t >= a.sinks)) return -1;
                const int blk = (int)block_of(c, a.b, cu.u.s, t, place);
                if (blk < 0) {
                    bad = true;
                    if constexpr (!TREE) report(c.status, kEInval);  // (mask_tree does)
                }
                return blk;
            };
            int place = 0;
            bool bad = false;
            int blk = look(place, bad);
            for (int x = 0, more = 1; more; ++x) {
                more = cu.more();
                const int h = cu.u.h, now = blk, at = place;
                const unsigned any = __ballot_sync(0xffffffffu, bad), boxes = __popc(__ballot_sync(0xffffffffu, now >= 0));
                if (more) {
                    cu.next(a, sh);
                    blk = look(place, bad);
                }
                if (!is_v) {
                    if (any && lane < 4) {  // a bit a box to a bit a token
                        uint32_t tokens = 0;
#pragma unroll 1
                        for (int k = 0; k < 32; ++k) tokens |= (any >> (lane * 32 + k) / box & 1) << k;
                        s_kbad[(x & 3) * 4 + lane] = tokens;
                    }
                    if (lane == 0) s_bad[x & 3] = any != 0;
                    bar_arrive_warp(sc_full + 8 * (x & 3));
                }
                const uint32_t st = item % kStages, round = item / kStages;
                item += 2;
                if (round > 0) ok = ok && bar_wait(kv_free + 8 * st, (round - 1) & 1, dead);
                if (!ok) continue;
                ++sent;
                const uint32_t bar = kv_full + 8 * st, to = smem_addr(tiles + st * S::kTile) + lane * box * 128;
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(boxes * box * 2 * DP) : "memory");
                __syncwarp();
                if (now >= 0) {
#pragma unroll
                    for (int p = 0; p < DP / 64; ++p)
                        asm volatile(
                            "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
                                to + p * S::kPanel), "l"(map), "r"(bar), "r"(p * 64), "r"(at), "r"(h), "r"(now)
                            : "memory");
                }
            }
            if (lane == 0) s_sent[is_v] = sent;
        } else if (warp >= S::kQueryWarp && warp < S::kQueryWarp + S::kQueryWarps) {
            // ================= queries to shared memory =================
            constexpr int QC = DP / 8, QS = S::kQueryWarps * 32 / QC;
            const int i = tid - S::kQueryWarp * 32, qc = i % QC;
            bool ok = true;
            for (int frag = 0;; ++frag) {
                const Unit &u = cu.u;
                if (i < 32) {
                    if (frag >= kJobs) ok = ok && bar_wait<true>(job_free + 8 * (frag % kJobs), (frag / kJobs - 1) & 1, dead);
                    if (ok && i == 0) {
                        Job &job = jobs[frag % kJobs];
                        job.u = u;
                        job.j0 = cu.j;
                        job.n = cu.end - cu.j;
                        job.whole = cu.whole();
                        job.last = cu.last;
                        job.c0 = job.c1 = job.slot = job.slot0 = 0;
                        if (!job.whole) {
                            job.c0 = cta_of(sh, cu.at + kWeight);
                            job.c1 = cta_of(sh, cu.at + kWeight + u.nt - 1);
                            job.slot = slot_of(sh, blockIdx.x, cu.at);
                            job.slot0 = slot_of(sh, job.c0, cu.at);
                        }
                        bar_arrive(job_full + 8 * (frag % kJobs));
                    }
                }
                __syncwarp();
                if (frag > 0) ok = ok && bar_wait<true>(q_free, (frag - 1) & 1, dead);
                if (ok && in.q_map) {
                    // by the copy engine, 128 rows of 64 elements at a time
                    if (lane == 0) {
                        const int halves = u.rows > 128 ? 2 : 1;
                        if (i == 0) {
                            s_sent[2] = frag + 1;
                            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(q_full), "r"(halves * S::kTile) : "memory");
                            for (int k = 0; k < halves; ++k)
                                for (int p = 0; p < DP / 64; ++p)
                                    asm volatile(
                                        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                                            smem_addr(smem) + k * S::kTile + p * S::kPanel), "l"(&in.q), "r"(q_full), "r"(p * 64), "r"(u.h * c.G),
                                        "r"(u.q0 + quot(u.qt * 256 + k * 128, c.div_g))
                                        : "memory");
                        } else {
                            bar_arrive(q_full);
                        }
                    }
                    __syncwarp();
                } else if (ok) {
#pragma unroll 4
                    for (int r = i / QC; r < 256; r += QS) {
                        const int gr = u.qt * 256 + r, t = quot(gr, c.div_g), hd = u.h * c.G + gr - t * c.G;
                        const bool real = r < u.rows && qc * 8 < c.D;
                        const int64_t at = real ? (int64_t)(u.q0 + t) * a.q_t + (int64_t)hd * a.q_h + qc * 16 : 0;
                        copy16(smem_addr(smem + r / 128 * S::kTile) + swizzled<DP>(r % 128, qc), a.q + at, real);
                    }
                    copy_commit();
                    copy_wait<0>();
                    shared_to_async();
                    bar_arrive_warp(q_full);
                }
                if (cu.last) break;
                cu.j = cu.end - 1;
                cu.next(a, sh);
            }
        } else if (warp == 8) {
            // ================= products: the warp waits, one thread issues =================
            const bool one = elect();
            constexpr uint32_t kQK = shape_of<BF16, kTok, false>(), kPV = shape_of<BF16, DP, true>();
            const uint32_t sq = smem_addr(smem), sk = smem_addr(tiles);
            uint32_t item = 0, n_p0 = 0, n_p1 = 0, n_o0 = 0, n_o1 = 0;
            bool ok = true;
            auto scores = [&](int h, uint32_t st) {
                if (!one) return;
                const uint64_t dq = operand(sq + h * S::kTile, 16), dk = operand(sk + st * S::kTile, 16);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    constexpr uint32_t kStep16 = 32 >> 4, kPanel16 = S::kPanel >> 4;  // addresses in the descriptor count 16 bytes
                    const uint32_t at = (k / 4) * kPanel16 + (k % 4) * kStep16;
                    mma_ss(tm + h * 128, dq + at, dk + at, kQK, k > 0);
                }
                commit(s_full + 8 * h);
            };
            auto full = [&](uint32_t it) { return bar_wait(kv_full + 8 * (it % kStages), it / kStages & 1, dead); };
            // one half's products of tile j: its sums, then its scores of the next tile
            auto half_tile = [&](int h, uint32_t &n_p, uint32_t &n_o, bool first, bool more, uint64_t dv, uint32_t st) {
                ok = bar_wait(p_half + 8 * h, n_p & 1, dead) && (!first || n_o == 0 || bar_wait(o_free + 8 * h, (n_o - 1) & 1, dead));
                if (!ok) return;
                after_sync();
                const uint32_t o = tm + 256 + h * 128, p = tm + h * 128 + 64;
                // the later half of the tokens first, as their weights come
                if (one)
#pragma unroll
                    for (int k = kTok / 32; k < kTok / 16; ++k) mma_ts(o, p + k * 8, dv + k * (2048 >> 4), kPV, !first || k > kTok / 32);
                __syncwarp();
                ok = bar_wait(p_full + 8 * h, n_p & 1, dead);
                if (!ok) return;
                after_sync();
                if (one) {
#pragma unroll
                    for (int k = 0; k < kTok / 32; ++k) mma_ts(o, p + k * 8, dv + k * (2048 >> 4), kPV, true);
                }
                if (more) scores(h, st);
                else if (one) commit(o_full + 8 * h);
                __syncwarp();
                ++n_p;
                n_o += !more;
            };
            for (int frag = 0; ok; ++frag) {
                ok = bar_wait(q_full, frag & 1, dead);
                if (!ok) break;
                const Job &job = jobs[frag % kJobs];
                const int n = job.n;
                const bool two = job.u.rows > 128, last = job.last;
                ok = full(item);
                if (!ok) break;
                after_sync();
                scores(0, item % kStages);
                if (two) scores(1, item % kStages);
                if (one) {
                    commit(kv_free + 8 * (item % kStages));
                    if (n == 1) commit(q_free);
                }
                __syncwarp();
                ++item;
                for (int j = 0; j < n && ok; ++j) {
                    const bool more = j + 1 < n;
                    const uint32_t sv = item % kStages, sk1 = (item + 1) % kStages;
                    ok = full(item) && (!more || full(item + 1));
                    if (!ok) break;
                    const uint64_t dv = operand(sk + sv * S::kTile, S::kPanel);
                    half_tile(0, n_p0, n_o0, j == 0, more, dv, sk1);
                    if (two && ok) half_tile(1, n_p1, n_o1, j == 0, more, dv, sk1);
                    if (!ok) break;
                    if (one) {
                        commit(kv_free + 8 * sv);
                        if (more) {
                            commit(kv_free + 8 * sk1);
                            if (j + 2 == n) commit(q_free);
                        }
                    }
                    __syncwarp();
                    item += more ? 2 : 1;
                }
                if (last) break;
            }
        }
        __syncwarp();
    }
    __syncthreads();
    if (*dead && warp == 8) {
        // the launch gave up: products and copies that were asked for end before their memory is given back (each wait
        // has a limit; a tile of K or V that another has followed in its stage is not waited for)
        auto over = [&](uint32_t bar, uint32_t parity) {
            for (uint32_t i = 0; i < kSpin / 64 && !bar_test(bar, parity); ++i) {
            }
        };
        if (elect()) commit(ended);  // (the thread that issued the products)
        __syncwarp();
        over(ended, 0);
        const uint32_t nk = s_sent[0], nv = s_sent[1];  // items 2 * (nk - 1) and 2 * nv - 1 are the last
        for (uint32_t st = 0; st < kStages; ++st) {
            uint32_t last = ~0u;
            for (uint32_t it = st; it < 2 * max(nk, nv); it += kStages)
                if (it / 2 < (it & 1 ? nv : nk)) last = it;
            if (last != ~0u) over(kv_full + 8 * st, last / kStages & 1);
        }
        if (s_sent[2]) over(q_full, (s_sent[2] - 1) & 1);
    }
    if (warp == 8) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
        if (lane == 0 && *dead) report(c.status, kECuda);
    }
    chain_next();
}

using Kernel = void (*)(const ChunkLaunch);
struct Pick {
    Kernel k;
    size_t smem;
    int threads;
};

template <int FMT, int DP, int LOAD, bool TREE>
Pick pick_type(bool bf16) {
    using S = Shape<DP, FMT, LOAD, TREE>;
    return {bf16 ? k_attend_chunk<true, FMT, DP, LOAD, TREE> : k_attend_chunk<false, FMT, DP, LOAD, TREE>, S::kSmem, S::kThreads};
}
template <int DP, bool TREE>
Pick pick_load(bool bf16, int fmt, bool tma) {
    return fmt == kFmtE4M3 ? pick_type<kFmtE4M3, DP, kConvert, TREE>(bf16)
         : fmt == kFmtInt8 ? pick_type<kFmtInt8, DP, kConvert, TREE>(bf16)
         : tma             ? pick_type<kFmt16, DP, kTma, TREE>(bf16)
                           : pick_type<kFmt16, DP, kGather, TREE>(bf16);
}
template <bool TREE>
Pick pick(bool bf16, int fmt, int D, bool tma) { return D <= 64 ? pick_load<64, TREE>(bf16, fmt, tma) : pick_load<128, TREE>(bf16, fmt, tma); }
template <bool TREE>
cudaError_t chunk_init() {
    for (int bf16 = 0; bf16 < 2; ++bf16)
        for (int load = 0; load < 4; ++load)
            for (int D = 64; D <= 128; D += 64) {
                const Pick p = pick<TREE>(bf16, load == 3 ? (int)kFmt16 : load, D, load == 3);
                const cudaError_t e = cudaFuncSetAttribute(p.k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem);
                if (e != cudaSuccess) return e;
            }
    return cudaSuccess;
}
template <bool TREE>
cudaError_t launch_chunk(const AttendLaunch &a, const CacheMaps &m, bool bf16, int fmt, int ctas, cudaStream_t st) {
    const Pick p = pick<TREE>(bf16, fmt, a.c.D, m.box > 0);
    ChunkLaunch l;
    l.a = a;
    l.m = m;
    l.q_map = 128 % a.c.G == 0 && encode_rows(a, bf16, l.q);
    return launch_chained(p.k, ctas, p.threads, p.smem, st, l);
}

}  // namespace

}  // namespace lr
