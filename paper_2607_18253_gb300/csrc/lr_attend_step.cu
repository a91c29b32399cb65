// Attention of few rows over a paged KV cache: the single tokens of many sequences.
//
// For the rows of a unit (lr_attend.cuh) the softmax needs one pass over the cached tokens: with
// the running maximum m, the sum l of exp(x_j - m) and the weighted sum o of v_j, a tile of tokens
// that raises m to m' scales l and o by exp(m - m') first.  Two ranges of tokens are
// joined the same way, so a unit may be split anywhere.
//
// What bounds it is the cache's bytes, and next to them the chain of dependent steps that a tile is: scores,
// maximum, weights, sums.  So the batch is one line of tiles, whatever sequences they belong to, of which
// each CTA takes an equal share (lr_attend.cuh), and within a CTA
//   - a tile's tokens are divided over the four warps, and a warp copies (cp.async, a tile or two ahead), waits
//     for and multiplies its own: nothing is exchanged until the unit ends, where the warps join their
//     sums through the stages just used, and the CTAs of a shared unit theirs through memory;
//   - the products are S^T = K Q^T and O^T += V^T P^T (16x8x16 tensor-core instructions): the 16-row operand is
//     the cache and the 8-column one the queries, so up to eight rows (NR = 1) cost half of what they would as half of
//     a 16-row operand, in instructions and registers, and more warps fit an SM;
//   - the maximum that the weights refer to lags behind the true one, so most tiles exchange nothing between lanes.
// Measured (32 query heads on 8 KV heads of 128, blocks of 16): a 16-bit cache 5.9 TB/s (63 sequences of
// 512 to 6,001 tokens, 96 us) and 4.8 (one of 200,001, 86 us: at the first rate its bytes are 69, the rest
// is the start and the join of 76 parts); e4m3 4.6 (64 of 128 to 8,192, 56 us), where a token is as many
// instructions as in 16 bits, and its conversion, for half the bytes: nothing is full (47% of issue slots, 56% of
// DRAM), the latency of a tile's steps at 12 warps an SM shows.
#include "lr_attend.cuh"

namespace lr {

namespace {

constexpr int kThreads = 128;
constexpr int kStepWeight = 2;  // tiles that a unit's beginning and end take the time of

// Where a 16-byte chunk of a cached vector lies in its shared-memory row, so that the eight rows that
// one instruction reads at a time are in different banks.
template <int DP, int FMT, bool V>
__device__ __forceinline__ int swizzle(int row, int chunk) {
    if constexpr (FMT == kFmt16) return chunk ^ (row & 7);
    else if constexpr (DP == 128) return V ? chunk ^ (row & 7) : chunk ^ ((row & 1) << 2);
    else return V ? chunk ^ (row >> 1 & 3) : chunk;
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DP, int FMT, int NR>
struct Solo {
    static constexpr int kRow = DP * (FMT == kFmt16 ? 2 : 1);
    static constexpr int kChunks = kRow / 16;
    static constexpr int kMine = FMT == kFmt16 ? 16 : 32;  // tokens of a warp
    static constexpr int kTile = 4 * kMine;
    static constexpr int kHalf = kMine * kRow;
    static constexpr int kStage = 2 * kHalf;
    // stages, and CTAs of an SM.  64 elements of 16 tokens in 4 CTAs; else by what the room takes, measured: 8-bit
    // 2 x 3 CTAs (256 sequences with a window over int8 131 us; 3 x 2: 150; 16 tokens, 3 x 4: 151), 16-bit
    // 3 x 2 (a context of 200,001 tokens 86 us; 2 x 3: 98).
    static constexpr int kStages = FMT == kFmt16 || DP == 64 ? 3 : 2;
    static constexpr int kCtas = NR == 2 ? 2 : DP == 64 ? (FMT == kFmt16 ? 4 : 3) : FMT == kFmt16 ? 2 : 3;
    static constexpr int kScales = FMT == kFmt16 ? 0 : kStages * 2 * kMine * 4;
    static constexpr int kWarp = kStages * kStage + kScales;
    static constexpr int kSmem = 4 * kWarp + 4 * 8 * NR * 8;
    static_assert(kStage >= 8 * NR * DP * 4, "room for a warp's sums");
};

// A part (m, l, sums) added to others whose common maximum is mm.
__device__ __forceinline__ void add_part(float2 ml, const float4 &w, float mm, float &ll, float4 &acc) {
    if (ml.x == -INFINITY && ml.y == 0.0f) return;  // saw nothing
    const float f = ml.x == -INFINITY ? 0.0f : exp2_fast(ml.x - mm);
    ll += ml.y == 0.0f ? 0.0f : ml.y * f;
    acc.x += w.x * f;
    acc.y += w.y * f;
    acc.z += w.z * f;
    acc.w += w.w * f;
}

// Elements d .. d + 3 of a finished row of a unit whose only tile of rows it is.
template <bool BF16>
__device__ __forceinline__ void write_row(const AttendLaunch &a, int r, int d, int q0, int h, float mm, float ll, float4 w) {
    const CacheDev &c = a.c;
    const int t = quot(r, c.div_g), hd = h * c.G + r - t * c.G;
    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
    if (d < c.D)
        *reinterpret_cast<uint2 *>(a.out + (int64_t)(q0 + t) * a.o_t + (int64_t)hd * a.o_h + d * 2) =
            make_uint2(pack16<BF16>(w.x * inv, w.y * inv), pack16<BF16>(w.z * inv, w.w * inv));
    if (a.lse && d == 0) a.lse[(int64_t)(q0 + t) * c.Hq + hd] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
}

// Joins the parts of a unit, in the order of the CTAs whichever came last: a warp a row, its lanes first the
// parts' maxima and sums, then four elements each of 16 parts at a time (of 2 x 16 with 64 elements).  The
// first part is in slot0, the others each the first of their CTAs.  (Not inlined: its registers are not the loop's.)
template <bool BF16, int DP>
__device__ __noinline__ void join_parts(const AttendLaunch &a, int c0, int parts, int slot0, int rows, int q0, int h) {
    constexpr int kLanes = DP / 4, kTwo = 32 / kLanes;
    const int lane = threadIdx.x % 32, part0 = lane / kLanes, e = lane % kLanes * 4;
    for (int r = threadIdx.x / 32; r < rows; r += kThreads / 32) {
        auto at = [&](int k) { return (int64_t)(k == 0 ? slot0 : 2 * (c0 + k)) * kStepRows + r; };
        float mm = -INFINITY, ll = 0.0f;
        for (int k = lane; k < parts; k += 32) mm = fmaxf(mm, __ldcg(&a.part_ml[at(k)].x));
#pragma unroll
        for (int z = 16; z >= 1; z /= 2) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, z));
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k0 = 0; k0 < parts; k0 += 16 * kTwo) {
            float2 ml = make_float2(-INFINITY, 0.0f);
            if (k0 + lane < parts && lane < 16 * kTwo) ml = __ldcg(a.part_ml + at(k0 + lane));
            float4 w[16];
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int k = k0 + z * kTwo + part0;
                w[z] = k < parts ? __ldcg(reinterpret_cast<const float4 *>(a.part_o + at(k) * 128 + e)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int src = z * kTwo + part0;
                add_part(make_float2(__shfl_sync(0xffffffffu, ml.x, src), __shfl_sync(0xffffffffu, ml.y, src)), w[z], mm, ll, acc);
            }
        }
        if constexpr (kTwo == 2) {
            ll += __shfl_xor_sync(0xffffffffu, ll, 16);
            acc.x += __shfl_xor_sync(0xffffffffu, acc.x, 16);
            acc.y += __shfl_xor_sync(0xffffffffu, acc.y, 16);
            acc.z += __shfl_xor_sync(0xffffffffu, acc.z, 16);
            acc.w += __shfl_xor_sync(0xffffffffu, acc.w, 16);
        }
        if (part0 == 0) write_row<BF16>(a, r, e, q0, h, mm, ll, acc);
    }
}

// Whether token t of a unit has a block out of range.
__device__ __forceinline__ bool no_block(const AttendLaunch &a, const Unit &u, int t) {
    int place;
    return t <= u.hi && block_of(a.c, a.b, u.s, t, place) < 0;
}

template <bool BF16, int FMT, int DP, int NR>
__global__ void __launch_bounds__(kThreads, Solo<DP, FMT, NR>::kCtas) k_attend_step(const __grid_constant__ AttendLaunch a) {
    using S = Solo<DP, FMT, NR>;
    constexpr int kRows = 8 * NR, kMine = S::kMine, NB = kMine / 16, KS = DP / 16;
    // 8-bit codes are multiplied in fp16, which holds them exactly and converts them in the fewest
    // instructions.  The queries come to fp16 as they are, or from bf16 divided by a power of two
    // a row that brings the largest to [1, 2): what fp16 then rounds is below 2^-24 of it.  The weights
    // carry V's scales, and are divided by a power of two a row that brings the largest such product of the tokens
    // that the row sees to [1, 16]: a large scale where the weight is small, or hidden, leaves the others what they are.
    constexpr bool MB = FMT == kFmt16 ? BF16 : false;  // type of the products
    // The maximum that the weights refer to is left behind until a score exceeds it by this (log2): any
    // reference gives the same quotient, and a tile that raises none needs no exchange between lanes.
    constexpr float kLag = MB ? 8.0f : 4.0f;
    extern __shared__ __align__(128) char smem[];
    __shared__ int s_last;
    __shared__ long long s_scratch[kThreads / 32 + 2];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, i4 = lane % 4;
    char *const stages = smem + warp * S::kWarp;
    float *const scales = reinterpret_cast<float *>(stages + S::kStages * S::kStage);  // [stage][K, V][token]
    float2 *const s_ml = reinterpret_cast<float2 *>(smem + 4 * S::kWarp);              // [warp][row]
    const CacheDev &c = a.c;

    chain_wait();
    Cursor<kRows, S::kTile, kStepWeight> cu, lk;
    Share sh;
    if (!take_share<kRows, S::kTile, kStepWeight, kThreads, 1>(a, cu, sh, s_scratch)) {
        chain_next();
        return;
    }
    lk = cu;
    bool ahead = true;  // lk stands at a tile that is to be requested

    // The block of lane l's token of the tile at lk, as the table has it: a load that nothing waits for until the
    // tile's copies are issued, a tile later.  Where blocks are multiples of 16 tokens, 16 neighbouring tokens
    // share one, and their addresses follow from the first's.  What no row of the unit sees is not looked up (its
    // block may be gone) and reads as zeros.
    const bool even = c.b % 16 == 0;
    int blk = -1, place = 0;
    auto seen = [&](int t) { return t <= lk.u.hi && !(a.window > 0 && t <= lk.u.lo - a.window && t >= a.sinks); };
    auto look = [&]() {
        const int t0 = lk.base() + warp * kMine, t = t0 + (even ? lane & ~15 : lane);
        const int i = quot(t, c.div_b);
        place = t - i * c.b;
        blk = -1;
        const int last = min(even ? t + 15 : t, lk.u.hi);
        const bool any = t <= lk.u.hi && (a.window == 0 || last > lk.u.lo - a.window || t < a.sinks);
        if (lane < kMine && any && i < a.b.max_blocks) blk = __ldg(a.b.table + (int64_t)lk.u.s * a.b.table_stride + i);
    };
    [[maybe_unused]] unsigned bad_tiles = 0;  // 16 bits: a bit for each tile on its way that has a block out of range
    auto issue = [&](int tile) {
        char *const st = stages + tile % S::kStages * S::kStage;
        constexpr int kStep = 32 / S::kChunks;
        const int ch = lane % S::kChunks, r0 = lane / S::kChunks, t0 = lk.base() + warp * kMine;
        const bool in = ch * 16 < c.D * (FMT == kFmt16 ? 2 : 1), mine = lane < kMine && seen(t0 + lane);
        const int myblk = even ? __shfl_sync(0xffffffffu, blk, lane & 16) : blk;
        const bool there = mine && (uint32_t)myblk < (uint32_t)c.nb;
        const unsigned have = __ballot_sync(0xffffffffu, there);  // a bit a token
        if (__any_sync(0xffffffffu, mine && !there)) {
            if constexpr (FMT == kFmt16) bad_tiles |= 1u << (tile & 31);
            report(c.status, kEInval);
        }
        if (even) {
#pragma unroll
            for (int r2 = 0; r2 < kMine; r2 += 16) {
                const int bk = __shfl_sync(0xffffffffu, blk, r2), pl = __shfl_sync(0xffffffffu, place, r2);
                int64_t at = (int64_t)bk * c.sb + (int64_t)(pl + r0) * c.st + lk.u.h * c.sh + ch * 16;
                const int64_t step = kStep * c.st;
#pragma unroll
                for (int r1 = r2; r1 < r2 + 16; r1 += kStep, at += step) {
                    const int r = r1 | r0;
                    const bool ok = in && (have >> r & 1);
                    const char *const k = ok ? c.k + at : c.k, *const v = ok ? c.v + at : c.v;
                    copy16(smem_addr(st + r * S::kRow + swizzle<DP, FMT, false>(r, ch) * 16), k, ok);
                    copy16(smem_addr(st + S::kHalf + r * S::kRow + swizzle<DP, FMT, true>(r, ch) * 16), v, ok);
                }
            }
        } else {
            const int64_t off = (int64_t)blk * c.sb + place * c.st + lk.u.h * c.sh + ch * 16;
#pragma unroll
            for (int r1 = 0; r1 < kMine; r1 += kStep) {
                const int r = r1 | r0;
                const int64_t o = __shfl_sync(0xffffffffu, off - ch * 16, r) + ch * 16;
                const bool ok = in && (have >> r & 1);
                const char *const k = ok ? c.k + o : c.k, *const v = ok ? c.v + o : c.v;
                copy16(smem_addr(st + r * S::kRow + swizzle<DP, FMT, false>(r, ch) * 16), k, ok);
                copy16(smem_addr(st + S::kHalf + r * S::kRow + swizzle<DP, FMT, true>(r, ch) * 16), v, ok);
            }
        }
        if constexpr (FMT != kFmt16) {
            if (lane < kMine) {
                const int64_t so = there ? (int64_t)myblk * c.ssb + (place + (even ? lane & 15 : 0)) * c.sst + lk.u.h * c.ssh : 0;
                float *const to = scales + tile % S::kStages * 2 * kMine + lane;
                copy4(smem_addr(to), there || !mine ? c.ks + so : c.nan, mine);  // (NaN where the block is out of range)
                copy4(smem_addr(to + kMine), c.vs + so, there);
            }
        }
    };
    look();
    for (int t = 0; t < S::kStages - 1; ++t) {
        if (ahead) {
            issue(t);
            ahead = lk.more();
            if (ahead) {
                lk.next(a, sh);
                look();
            }
        }
        copy_commit();
    }

    // a lane's columns are the rows n * 8 + 2 * i4, + 1 of the unit
    uint32_t q[KS][NR][2];
    float o[KS][NR][4], m[NR][2], l[NR][2], qf[NR][2], less[NR][2];  // less: m, 0 where it is -inf
    [[maybe_unused]] float down[NR][2];  // 8 bits: the power of two that the row's weights are multiplied by
    int pos[NR][2];
    for (int x = 0;;) {
        const Unit &u = cu.u;
        const bool whole = cu.whole(), last_unit = cu.last;
        {  // its queries, straight to the registers that multiply them
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const int r = n * 8 + g;  // (the row whose elements the lane holds)
                const int t = quot(r, c.div_g), hd = r - t * c.G;
                const bool ok = r < u.rows;
                const char *const p = a.q + (int64_t)(u.q0 + t) * a.q_t + (int64_t)(u.h * c.G + hd) * a.q_h;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if constexpr (FMT == kFmt16) {
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int d = k * 16 + z * 8 + 2 * i4;
                            q[k][n][z] = ok && d < c.D ? __ldg(reinterpret_cast<const uint32_t *>(p + d * 2)) : 0u;
                        }
                    } else {  // four neighbouring elements, the order in which the codes lie in a register
                        const int d = (k / 4) * 64 + i4 * 16 + (k % 4) * 4;
                        const uint2 w = ok && d < c.D ? __ldg(reinterpret_cast<const uint2 *>(p + d * 2)) : make_uint2(0, 0);
                        q[k][n][0] = w.x;
                        q[k][n][1] = w.y;
                    }
#pragma unroll
                    for (int z = 0; z < 4; ++z) o[k][n][z] = 0.0f;
                }
                float pow2 = 1.0f;
                if constexpr (FMT != kFmt16 && BF16) {
                    float top = 0.0f;
#pragma unroll
                    for (int k = 0; k < 2 * KS; ++k) {
                        const float2 f = unpack16<true>(q[k / 2][n][k % 2]);
                        top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // (not below 2^-100, whose reciprocal is a number; infinities stay what they are)
                    const uint32_t e = min(max(__float_as_uint(top) & 0x7f800000u, 27u << 23), 253u << 23);
                    const float inv = __uint_as_float((254u << 23) - e);
                    pow2 = __uint_as_float(e);
#pragma unroll
                    for (int k = 0; k < 2 * KS; ++k) {
                        const float2 f = unpack16<true>(q[k / 2][n][k % 2]);
                        q[k / 2][n][k % 2] = pack16<false>(f.x * inv, f.y * inv);
                    }
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int row = n * 8 + 2 * i4 + y;
                    pos[n][y] = row < u.rows ? u.kv - u.ql + quot(row, c.div_g) : -1;
                    qf[n][y] = a.scale_log2 * __shfl_sync(0xffffffffu, pow2, (2 * i4 + y) * 4);
                    m[n][y] = -INFINITY;
                    less[n][y] = 0.0f;
                    l[n][y] = 0.0f;
                    down[n][y] = 1.0f;
                }
            }
        }
        for (; cu.j < cu.end; ++x, ++cu.j) {
            // the copies of the tile ahead, then the places of the one after it (their latency is the tile's work)
            if (ahead) {
                issue(x + S::kStages - 1);
                ahead = lk.more();
                if (ahead) {
                    lk.next(a, sh);
                    look();
                }
            }
            copy_commit();
            copy_wait<S::kStages - 1>();
            __syncwarp();

            // ---- scores: tokens g, g + 8 of each 16 ----
            char *const st = stages + x % S::kStages * S::kStage;
            const uint32_t sk = smem_addr(st), sv = sk + S::kHalf;
            const int base = cu.base() + warp * kMine;
            if constexpr (FMT == kFmt16) {
                if (bad_tiles >> (x & 31) & 1) {  // K of a token whose block is out of range: NaN, as are its scores where a row sees them
                    bad_tiles &= ~(1u << (x & 31));
                    if (lane < kMine && no_block(a, u, base + lane))
                        *reinterpret_cast<uint16_t *>(st + lane * S::kRow + swizzle<DP, FMT, false>(lane, 0) * 16) = 0x7fff;
                    __syncwarp();
                }
            }
            float s[NB][NR][4];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int z = 0; z < 4; ++z) s[b][n][z] = 0.0f;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (FMT == kFmt16) {
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        uint32_t w[4];
                        const int row = b * 16 + lane % 16;
                        ldsm4(w, sk + row * S::kRow + swizzle<DP, FMT, false>(row, k * 2 + lane / 16) * 16);
#pragma unroll
                        for (int n = 0; n < NR; ++n) mma<MB>(s[b][n], w, q[k][n][0], q[k][n][1]);
                    }
                } else {
#pragma unroll
                    for (int hf = 0; hf < DP / 64; ++hf) {
                        const int row = b * 16 + g;
                        const uint4 w = lds16(sk + row * S::kRow + swizzle<DP, FMT, false>(row, hf * 4 + i4) * 16);
                        const uint4 v = lds16(sk + (row + 8) * S::kRow + swizzle<DP, FMT, false>(row + 8, hf * 4 + i4) * 16);
                        const uint32_t ww[4] = {w.x, w.y, w.z, w.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t f[4];
                            to_half<FMT, false>(ww[k], f[0], f[2]);
                            to_half<FMT, false>(vv[k], f[1], f[3]);
#pragma unroll
                            for (int n = 0; n < NR; ++n) mma<MB>(s[b][n], f, q[hf * 4 + k][n][0], q[hf * 4 + k][n][1]);
                        }
                    }
                }
            }
            // ---- softmax ----
            const float *const ks = scales + x % S::kStages * 2 * kMine, *const vs = ks + kMine;
            const bool masked = base + kMine - 1 > u.lo || (a.window > 0 && base <= u.hi - a.window && base + kMine > a.sinks);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        float f = qf[n][z & 1];
                        if constexpr (FMT != kFmt16) f *= ks[b * 16 + g + (z >> 1) * 8];
                        s[b][n][z] *= f;
                    }
            if (masked) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int z = 0; z < 4; ++z)
                            if (!visible(pos[n][z & 1], base + b * 16 + g + (z >> 1) * 8, a.window, a.sinks)) s[b][n][z] = -INFINITY;
            }
            float mx[NR][2];
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    mx[n][y] = fmaxf(s[0][n][y], s[0][n][y + 2]);
#pragma unroll
                    for (int b = 1; b < NB; ++b) mx[n][y] = fmaxf(mx[n][y], fmaxf(s[b][n][y], s[b][n][y + 2]));
                    raise |= mx[n][y] > m[n][y] + kLag;
                }
            const bool raised = __any_sync(0xffffffffu, raise);
            [[maybe_unused]] float fo[NR][2];
            if constexpr (FMT != kFmt16) {
#pragma unroll
                for (int n = 0; n < NR; ++n) fo[n][0] = fo[n][1] = 1.0f;
            }
            if (raised) {
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        float w = mx[n][y];
                        w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 4));
                        w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 8));
                        w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 16));
                        const float mn = fmaxf(m[n][y], w), f = mn == -INFINITY ? 1.0f : exp2_fast(m[n][y] - mn);
                        m[n][y] = mn;
                        less[n][y] = mn == -INFINITY ? 0.0f : mn;
                        l[n][y] *= f;
                        if constexpr (FMT == kFmt16) {
#pragma unroll
                            for (int k = 0; k < KS; ++k) {
                                o[k][n][y] *= f;
                                o[k][n][y + 2] *= f;
                            }
                        } else {
                            fo[n][y] = f;
                        }
                    }
            }
            [[maybe_unused]] float wx[NR][2];
            if constexpr (FMT != kFmt16) {
#pragma unroll
                for (int n = 0; n < NR; ++n) wx[n][0] = wx[n][1] = 0.0f;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const float p = exp2_fast(s[b][n][z] - less[n][z & 1]);
                        l[n][z & 1] += p;
                        if constexpr (FMT != kFmt16) {
                            // (a scale that is not finite stays away from a weight that the mask takes)
                            const float w = p * vs[b * 16 + g + (z >> 1) * 8];
                            s[b][n][z] = masked && s[b][n][z] == -INFINITY ? 0.0f : w;
                            wx[n][z & 1] = fmaxf(wx[n][z & 1], fabsf(s[b][n][z]));
                        } else {
                            s[b][n][z] = p;
                        }
                    }
            if constexpr (FMT != kFmt16) {
                bool grow = raised;
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int y = 0; y < 2; ++y) grow |= wx[n][y] * down[n][y] > 16.0f;
                if (__any_sync(0xffffffffu, grow)) {
                    constexpr uint32_t kOne = 127u << 23, kFar = 120u << 23;
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float w = wx[n][y];
                            w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 4));
                            w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 8));
                            w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, 16));
                            // the largest product so far against the maximum as it is now, and its power of two
                            const float was = fo[n][y] * __uint_as_float(2 * kOne - __float_as_uint(down[n][y]));
                            const uint32_t e = __float_as_uint(fmaxf(was, w)) & 0x7f800000u;
                            down[n][y] = __uint_as_float(2 * kOne - min(max(e, kOne - kFar), kOne + kFar));
                            const float f = was * down[n][y];  // at most 2: no part of it overflows
#pragma unroll
                            for (int k = 0; k < KS; ++k) {
                                o[k][n][y] *= f;
                                o[k][n][y + 2] *= f;
                            }
                        }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int z = 0; z < 4; ++z) s[b][n][z] *= down[n][z & 1];
            }

            // ---- weighted sum ----
            bool slow = false;
            if constexpr (FMT == kFmt16) {
                // an infinity or a NaN in V that some row may not see: 0 times it is not 0, so such a tile is
                // summed without the tensor cores, skipping what a row does not see
                if (masked) {
                    bool z = false;
                    for (int k = lane; k < kMine * S::kChunks; k += 32) {
                        const uint4 w = lds16(sv + k * 16);
                        z |= not_finite<BF16>(w.x) || not_finite<BF16>(w.y) || not_finite<BF16>(w.z) || not_finite<BF16>(w.w);
                    }
                    slow = __any_sync(0xffffffffu, z);
                }
            }
            if (!slow) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    // the weights turned, from a lane's token to a lane's row
                    uint32_t p[NR][2];
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(p[n][y]) : "r"(pack16<MB>(s[b][n][2 * y], s[b][n][2 * y + 1])));
                    const int mi = lane / 8;
                    if constexpr (FMT == kFmt16) {
#pragma unroll
                        for (int k = 0; k < KS; ++k) {
                            uint32_t w[4];
                            const int row = b * 16 + (mi >> 1) * 8 + lane % 8;
                            ldsm4t(w, sv + row * S::kRow + swizzle<DP, FMT, true>(row, k * 2 + (mi & 1)) * 16);
#pragma unroll
                            for (int n = 0; n < NR; ++n) mma<MB>(o[k][n], w, p[n][0], p[n][1]);
                        }
                    } else {
                        // pairs of neighbouring elements move as one: rows g of the product are the even ones of 16, rows
                        // g + 8 the odd ones
#pragma unroll
                        for (int k = 0; k < KS; k += 2) {
                            uint32_t w[4];
                            const int row = b * 16 + (mi & 1) * 8 + lane % 8;
                            ldsm4t(w, sv + row * S::kRow + swizzle<DP, FMT, true>(row, k + (mi >> 1)) * 16);
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (FMT == kFmtE4M3 && masked) {  // codes of NaN stay away from weights that the mask takes
                                    w[2 * e] = without_nan(w[2 * e]);
                                    w[2 * e + 1] = without_nan(w[2 * e + 1]);
                                }
                                uint32_t f[4];
                                to_half<FMT, true>(w[2 * e], f[0], f[1]);
                                to_half<FMT, true>(w[2 * e + 1], f[2], f[3]);
#pragma unroll
                                for (int n = 0; n < NR; ++n) mma<MB>(o[k + e][n], f, p[n][0], p[n][1]);
                            }
                        }
                    }
                }
            } else if constexpr (FMT == kFmt16) {
                for (int t = 0; t < kMine; ++t) {
                    const int src = (t & 7) * 4 + i4;
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        float w[2];
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const float e0 = __shfl_sync(0xffffffffu, s[0][n][y], src), e1 = __shfl_sync(0xffffffffu, s[0][n][y + 2], src);
                            w[y] = unpack16<BF16>(pack16<BF16>(t & 8 ? e1 : e0, 0.0f)).x;
                        }
                        const bool v0 = visible(pos[n][0], base + t, a.window, a.sinks), v1 = visible(pos[n][1], base + t, a.window, a.sinks);
#pragma unroll
                        for (int k = 0; k < KS; ++k)
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const float v = unpack16<BF16>(*reinterpret_cast<const uint16_t *>(
                                    st + S::kHalf + t * S::kRow + swizzle<DP, FMT, true>(t, k * 2 + y) * 16 + g * 2)).x;
                                if (v0) o[k][n][2 * y] += w[0] * v;
                                if (v1) o[k][n][2 * y + 1] += w[1] * v;
                            }
                    }
                }
            }
            __syncwarp();
        }

        // ---- the unit ends here, for this CTA: the warps' sums to their stages just used, [row][element] ----
        const int used = (x - 1) % S::kStages * S::kStage;
        float *const xo = reinterpret_cast<float *>(stages + used);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float w = l[n][y];
                w += __shfl_xor_sync(0xffffffffu, w, 4);
                w += __shfl_xor_sync(0xffffffffu, w, 8);
                w += __shfl_xor_sync(0xffffffffu, w, 16);
                const int r = n * 8 + 2 * i4 + y;
                if (r >= u.rows) continue;
                if (g == 0) s_ml[warp * kRows + r] = make_float2(m[n][y], w);
                const float f = FMT == kFmt16 ? 1.0f : __uint_as_float((254u << 23) - __float_as_uint(down[n][y]));
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    if constexpr (FMT == kFmt16) {
                        xo[r * DP + k * 16 + g] = o[k][n][y];
                        xo[r * DP + k * 16 + g + 8] = o[k][n][y + 2];
                    } else {
                        *reinterpret_cast<float2 *>(xo + r * DP + k * 16 + 2 * g) = make_float2(o[k][n][y] * f, o[k][n][y + 2] * f);
                    }
                }
            }
        __syncthreads();
        constexpr int kLanes = DP / 4;  // four elements a thread
        const int d = tid % kLanes * 4;
        int64_t slot = 0;
        if (!whole) slot = slot_of(sh, blockIdx.x, cu.at);
        for (int r = tid / kLanes; r < u.rows; r += kThreads / kLanes) {
            float mm = -INFINITY, ll = 0.0f;
            float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_ml[w * kRows + r].x);
#pragma unroll
            for (int w = 0; w < 4; ++w)
                add_part(s_ml[w * kRows + r], *reinterpret_cast<const float4 *>(smem + w * S::kWarp + used + (r * DP + d) * 4), mm, ll, acc);
            if (whole) {
                write_row<BF16>(a, r, d, u.q0, u.h, mm, ll, acc);
            } else {
                if (d == 0) a.part_ml[slot * kStepRows + r] = make_float2(mm, ll);
                *reinterpret_cast<float4 *>(a.part_o + (slot * kStepRows + r) * 128 + d) = acc;
            }
        }
        if (!whole) {
            const int c0 = cta_of(sh, cu.at + kStepWeight), c1 = cta_of(sh, cu.at + kStepWeight + u.nt - 1);
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const bool last = atomicAdd(a.done + c0, 1u) == (uint32_t)(c1 - c0);
                if (last) a.done[c0] = 0;
                s_last = last;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                join_parts<BF16, DP>(a, c0, c1 - c0 + 1, slot_of(sh, c0, cu.at), u.rows, u.q0, u.h);
            }
        }
        __syncthreads();  // the stages are free again
        if (last_unit) break;
        --cu.j;  // (the last tile that was taken)
        cu.next(a, sh);
    }
    chain_next();
}

using Kernel = void (*)(const AttendLaunch);
struct Pick {
    Kernel k;
    size_t smem;
    int ctas;  // of an SM
};

template <bool BF16, int FMT, int DP>
Pick pick_rows(int rows) {
    if (rows <= 8) return {k_attend_step<BF16, FMT, DP, 1>, Solo<DP, FMT, 1>::kSmem, Solo<DP, FMT, 1>::kCtas};
    return {k_attend_step<BF16, FMT, DP, 2>, Solo<DP, FMT, 2>::kSmem, Solo<DP, FMT, 2>::kCtas};
}
template <int FMT>
Pick pick_type(bool bf16, int D, int rows) {
    return D <= 64 ? (bf16 ? pick_rows<true, FMT, 64>(rows) : pick_rows<false, FMT, 64>(rows))
                   : (bf16 ? pick_rows<true, FMT, 128>(rows) : pick_rows<false, FMT, 128>(rows));
}
Pick pick(bool bf16, int fmt, int D, int rows) {
    return fmt == kFmt16 ? pick_type<kFmt16>(bf16, D, rows)
         : fmt == kFmtE4M3 ? pick_type<kFmtE4M3>(bf16, D, rows)
                           : pick_type<kFmtInt8>(bf16, D, rows);
}

}  // namespace

int attend_step_ctas(int sms) { return 4 * sms; }

cudaError_t attend_step_init() {
    for (int bf16 = 0; bf16 < 2; ++bf16)
        for (int fmt = 0; fmt < 3; ++fmt)
            for (int D = 64; D <= 128; D += 64)
                for (int rows = 8; rows <= 16; rows *= 2) {
                    const Pick p = pick(bf16, fmt, D, rows);
                    const cudaError_t e = cudaFuncSetAttribute(p.k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem);
                    if (e != cudaSuccess) return e;
                }
    return cudaSuccess;
}

cudaError_t launch_attend_step(const AttendLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st) {
    const Pick p = pick(bf16, fmt, a.c.D, rows);
    return launch_chained(p.k, p.ctas * sms, kThreads, p.smem, st, a);
}

}  // namespace lr
