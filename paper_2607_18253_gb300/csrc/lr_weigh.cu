// Attention weight that cached tokens have received, from the rows of a batch.
//
// With the rows' lse known, a weight needs no running maximum: w[j] += sum_r exp(scale q_r . k_j - lse_r).  A token's sum
// stays with the warp that has the token, so nothing is joined and the order of the sum is the rows' own.
//
// What bounds it for few rows is K's bytes.  Sixteen (or 32, 64) tokens are a warp's at a time; a lane reads 16-byte pieces of
// the vectors of tokens g and g + 8 straight to the registers that multiply them (S = K Q^T, 16x8x16 products with the cache as
// the 16-row operand): which elements of a vector a product sums is free, as long as the queries' lanes
// take the same ones, so a piece is two (16 bits) or four (8 bits) products' operands as it lies.  The next tokens'
// blocks are looked up while these are multiplied; their reads are other warps' to hide.
// Measured (64 single tokens over 128 to 8,192, 32 query heads on 8 KV heads of 128, e4m3): 50 us, 2.75 TB/s.  DRAM is a third busy and
// the issue slots 40%: what bounds it is a warp's own chain of conversions and dependent steps.  Vectors asked for a tile ahead (to
// the L2 cache) 54 us, five CTAs an SM, which spill, 68, heads in turn instead of tiles (queries loaded anew each) 83.  Over 16 bits, with
// nothing to convert, five CTAs do not spill (caches cold: 69 us, 3.8 TB/s, where four take 75; 256 sequences 139 and 157; one token over
// 60,000 42 and 46).
#include <algorithm>

#include "lr_attend.cuh"

namespace lr {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;

template <int DP, int FMT, int NR>
struct Piece {
    static constexpr int kVec = DP * (FMT == kFmt16 ? 2 : 1) / 64;  // 16-byte pieces a lane and vector
    static constexpr int NB = 4 / kVec;                             // blocks of 16 tokens
    static constexpr int kTile = 16 * NB;
    static constexpr int kCtas = NR == 1 && FMT == kFmt16 ? 5 : 4;                   // of an SM
};

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// (of a number: an infinity's two products need not have the same sign)
__device__ __forceinline__ float lse_log2(const WeighLaunch &a, float l) { return fmaf(l, a.lse_log2, l * a.lse_log2_rest); }

// The batch's tiles of tokens in one line: sequences in order, in a sequence head after head, so that a warp keeps its queries
// from tile to tile.  What no row sees is left out where nothing changes it.
template <int TILE>
struct Walk {
    int s, q0, ql, kv;
    int ns, wf, nt;  // tiles of sinks before the window, the window's first tile, tiles in all
    int tile, h;
    __device__ __forceinline__ bool load(const WeighLaunch &a) {
        if (!load_seq(a.a, s, q0, ql, kv) || kv == 0) return false;
        if (a.decay == 1.0f) nt = tile_count<TILE>(kv - ql, kv - 1, a.a.window, a.a.sinks, ns, wf);
        else ns = wf = 0, nt = (kv - 1) / TILE + 1;
        return true;
    }
    // On by so many tiles; false behind the last sequence.
    __device__ __forceinline__ bool on(const WeighLaunch &a, int tiles) {
        tile += tiles;
        while (tile >= nt) {
            tile -= nt;
            if (++h < a.a.c.H) continue;
            h = 0;
            do
                if (++s >= a.a.b.n) return false;
            while (!load(a));
        }
        return true;
    }
    __device__ __forceinline__ int base() const { return (tile < ns ? tile : wf + tile - ns) * TILE; }
};

template <bool BF16, int FMT, int DP, int NR, bool EVEN>
__global__ void __launch_bounds__(kThreads, Piece<DP, FMT, NR>::kCtas) k_weigh_step(const __grid_constant__ WeighLaunch a) {
    using P = Piece<DP, FMT, NR>;
    constexpr int kRows = 8 * NR, NB = P::NB, KS = DP / 16;
    // 8-bit codes are multiplied in fp16, which holds them exactly; bf16 queries come to it divided by a power of two a row
    // that brings the largest to [1, 2): what fp16 then rounds is below 2^-24 of it.
    constexpr bool MB = FMT == kFmt16 ? BF16 : false;
    __shared__ long long s_sum[kWarps], s_at;
    __shared__ int s_seq;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, i4 = lane % 4;
    const CacheDev &c = a.a.c;
    chain_wait();

    // this CTA's share of the line, x0 .. x1
    const int n = a.a.b.n;
    Walk<P::kTile> at;
    auto tiles_of = [&](int s) -> long long {
        at.s = s;
        return s < n && at.load(a) ? (long long)at.nt * c.H : 0;
    };
    long long all = 0, mine = 0, incl = 0;
    for (int base = 0; base < n; base += kThreads) {
        mine = tiles_of(base + tid);
        long long t;
        incl = block_sum<kThreads>(mine, s_sum, t);
        all += t;
    }
    const long long x0 = all * blockIdx.x / gridDim.x, x1 = all * (blockIdx.x + 1) / gridDim.x;
    if (x0 >= x1) {
        chain_next();
        return;
    }
    long long first = 0;
    for (int base = 0; base < n; base += kThreads) {
        long long t = all;
        if (n > kThreads) {
            mine = tiles_of(base + tid);
            incl = block_sum<kThreads>(mine, s_sum, t);
        }
        const long long x = x0 - first;
        if (x < incl && x >= incl - mine) {
            s_seq = base + tid;
            s_at = x - (incl - mine);
        }
        first += t;
        if (first > x0) break;
    }
    __syncthreads();
    at.s = s_seq;
    at.load(a);
    at.h = (int)(s_at / at.nt);
    at.tile = (int)(s_at - (long long)at.h * at.nt);
    if (x0 + warp >= x1 || !at.on(a, warp)) {
        chain_next();
        return;
    }

    // The blocks of a lane's tokens (g and g + 8 of each 16), as the table has them: looked up a tile ahead.  Where blocks are
    // multiples of 16 tokens, the 16 share one, and their addresses follow from the first's.
    constexpr int kLooks = EVEN ? 1 : 2;
    int blk[NB][kLooks];
    auto look = [&]() {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int y = 0; y < kLooks; ++y) {
                const int t = at.base() + b * 16 + (EVEN ? 0 : y * 8 + g), i = quot(t, c.div_b);
                blk[b][y] = t < at.kv && i < a.a.b.max_blocks ? __ldg(a.a.b.table + (int64_t)at.s * a.a.b.table_stride + i) : -1;
            }
    };
    look();
    uint32_t q[KS][NR][2];
    float qf[NR][2], less[NR][2];  // the scores' factor, lse * log2(e)
    int pos[NR][2];                // the rows' positions, -1: none
    int qh = -1, qs = -1, qr = -1;  // whose queries these are
    long long left = (x1 - x0 - warp + kWarps - 1) / kWarps;
    while (left-- > 0) {
        const int q0 = at.q0, ql = at.ql, kv = at.kv, h = at.h, tile0 = at.base();
        const int lo = kv - ql, rows = ql * c.G, end = tile0 + P::kTile - 1;
        uint4 k[NB][2][P::kVec];
        [[maybe_unused]] float ks[NB][2];
        int64_t to[NB];  // where this lane's token's weight is, -1: not this lane's to write
        float old[NB], sum[NB][2];
        // (no window hides a token of the tile, and it has no end: nearly always)
        const bool full = end < kv && !(a.a.window > 0 && tile0 <= lo - a.a.window && end >= a.a.sinks);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            to[b] = -1;
            old[b] = sum[b][0] = sum[b][1] = 0.0f;
            [[maybe_unused]] const int t16 = tile0 + b * 16, place16 = EVEN ? t16 - quot(t16, c.div_b) * c.b + g : 0;
            [[maybe_unused]] const char *const p16 = EVEN ? c.k + (int64_t)blk[b][0] * c.sb + place16 * c.st + h * c.sh + i4 * 16 : nullptr;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int t = tile0 + b * 16 + y * 8 + g, bk = blk[b][EVEN ? 0 : y];
                const int place = EVEN ? place16 + y * 8 : t - quot(t, c.div_b) * c.b;
                const bool any = full || !(a.a.window > 0 && t <= lo - a.a.window && t >= a.a.sinks);  // (some row sees it)
                bool ok = full || (t < kv && (any || a.decay != 1.0f));
                if (ok && (uint32_t)bk >= (uint32_t)c.nb) {  // (a token that no row sees may have no block any more)
                    if (any) report(c.status, kEInval);
                    ok = false;
                }
                const char *const p = EVEN ? p16 + y * 8 * c.st : c.k + (int64_t)bk * c.sb + place * c.st + h * c.sh + i4 * 16;
#pragma unroll
                for (int v = 0; v < P::kVec; ++v) {
                    const int e = (v * 4 + i4) * 16;
                    k[b][y][v] = make_uint4(0, 0, 0, 0);
                    if (ok && any && e < c.D * (FMT == kFmt16 ? 2 : 1)) k[b][y][v] = __ldg(reinterpret_cast<const uint4 *>(p + v * 64));
                }
                if constexpr (FMT != kFmt16) ks[b][y] = ok && any ? __ldg(c.ks + (int64_t)bk * c.ssb + place * c.sst + h * c.ssh) : 0.0f;
                if (ok && i4 == y) {
                    to[b] = (int64_t)bk * a.wb + place * a.wt + h * a.wh;
                    if (a.decay != 0.0f && t < lo) old[b] = a.decay * a.w[to[b]];
                }
            }
        }
        if (left > 0 && at.on(a, kWarps)) look();
        // rows from the first that may see the tile on; below a window, up to the last
        int r0 = tile0 > lo ? (tile0 - lo) * c.G / kRows * kRows : 0, r1 = rows;
        if (a.a.window > 0 && tile0 >= a.a.sinks) r1 = (int)min((long long)rows, max(0ll, (long long)end + a.a.window - lo) * c.G);
        for (; r0 < r1; r0 += kRows) {
            if (h != qh || q0 != qs || r0 != qr) {
                qh = h, qs = q0, qr = r0;
#pragma unroll
                for (int m = 0; m < NR; ++m) {
                    const int r = r0 + m * 8 + g;  // (the row whose elements the lane holds)
                    const int t = quot(r, c.div_g), hd = r - t * c.G;
                    const bool ok = r < rows;
                    const char *const p = a.a.q + (int64_t)(q0 + t) * a.a.q_t + (int64_t)(h * c.G + hd) * a.a.q_h;
                    float pow2 = 1.0f;
                    if constexpr (FMT == kFmt16) {
#pragma unroll
                        for (int v = 0; v < P::kVec; ++v) {
                            const int d = (v * 4 + i4) * 8;
                            const uint4 w = ok && d < c.D ? __ldg(reinterpret_cast<const uint4 *>(p + d * 2)) : make_uint4(0, 0, 0, 0);
                            q[2 * v][m][0] = w.x;
                            q[2 * v][m][1] = w.y;
                            q[2 * v + 1][m][0] = w.z;
                            q[2 * v + 1][m][1] = w.w;
                        }
                    } else {
#pragma unroll
                        for (int v = 0; v < P::kVec; ++v)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const int d = (v * 4 + i4) * 16 + u * 8;
                                const uint4 w = ok && d < c.D ? __ldg(reinterpret_cast<const uint4 *>(p + d * 2)) : make_uint4(0, 0, 0, 0);
                                q[4 * v + 2 * u][m][0] = w.x;
                                q[4 * v + 2 * u][m][1] = w.y;
                                q[4 * v + 2 * u + 1][m][0] = w.z;
                                q[4 * v + 2 * u + 1][m][1] = w.w;
                            }
                        if constexpr (BF16) {
                            float top = 0.0f;
#pragma unroll
                            for (int k = 0; k < 2 * KS; ++k) {
                                const float2 f = unpack16<true>(q[k / 2][m][k % 2]);
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
                                const float2 f = unpack16<true>(q[k / 2][m][k % 2]);
                                q[k / 2][m][k % 2] = pack16<false>(f.x * inv, f.y * inv);
                            }
                        }
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int row = r0 + m * 8 + 2 * i4 + y, tt = quot(row, c.div_g);
                        const bool real = row < rows;
                        const float l = real ? __ldg(a.a.lse + (int64_t)(q0 + tt) * c.Hq + h * c.G + row - tt * c.G) : -INFINITY;
                        // (a row that saw nothing adds nothing; one with an lse of +inf neither, as exp(x - inf))
                        const bool none = fabsf(l) == INFINITY;
                        pos[m][y] = none ? -1 : lo + tt;
                        less[m][y] = none ? 0.0f : lse_log2(a, l);
                        qf[m][y] = a.a.scale_log2 * __shfl_sync(0xffffffffu, pow2, (2 * i4 + y) * 4);
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float s[NR][4];
#pragma unroll
                for (int m = 0; m < NR; ++m)
#pragma unroll
                    for (int z = 0; z < 4; ++z) s[m][z] = 0.0f;
#pragma unroll
                for (int v = 0; v < P::kVec; ++v) {
                    const uint4 e = k[b][0][v], f = k[b][1][v];
                    const uint32_t ee[4] = {e.x, e.y, e.z, e.w}, ff[4] = {f.x, f.y, f.z, f.w};
                    if constexpr (FMT == kFmt16) {
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int m = 0; m < NR; ++m)
                                mma<MB>(s[m], ee[2 * u], ff[2 * u], ee[2 * u + 1], ff[2 * u + 1], q[2 * v + u][m][0], q[2 * v + u][m][1]);
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            uint32_t f0, f1, f2, f3;
                            to_half<FMT, false>(ee[u], f0, f2);
                            to_half<FMT, false>(ff[u], f1, f3);
#pragma unroll
                            for (int m = 0; m < NR; ++m) mma<MB>(s[m], f0, f1, f2, f3, q[4 * v + u][m][0], q[4 * v + u][m][1]);
                        }
                    }
                }
                const bool masked = !full || end > lo || (a.a.window > 0 && tile0 <= kv - 1 - a.a.window && end >= a.a.sinks);
#pragma unroll
                for (int m = 0; m < NR; ++m)
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        float f = qf[m][z & 1];
                        if constexpr (FMT != kFmt16) f *= ks[b][z >> 1];
                        s[m][z] = exp2_fast(s[m][z] * f - less[m][z & 1]);
                    }
                if (masked) {
#pragma unroll
                    for (int m = 0; m < NR; ++m)
#pragma unroll
                        for (int z = 0; z < 4; ++z)
                            if (!visible(pos[m][z & 1], tile0 + b * 16 + (z >> 1) * 8 + g, a.a.window, a.a.sinks)) s[m][z] = 0.0f;
                }
#pragma unroll
                for (int m = 0; m < NR; ++m)
#pragma unroll
                    for (int z = 0; z < 4; ++z) sum[b][z >> 1] += pos[m][z & 1] >= 0 ? s[m][z] : 0.0f;
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float f = sum[b][y];
                f += __shfl_xor_sync(0xffffffffu, f, 1);
                f += __shfl_xor_sync(0xffffffffu, f, 2);
                if (i4 == y && to[b] >= 0) a.w[to[b]] = old[b] + f;
            }
    }
    chain_next();
}

using Kernel = void (*)(const WeighLaunch);
template <int FMT, int DP, int NR>
Kernel pick_even(bool bf16, bool even) {
    return even ? (bf16 ? k_weigh_step<true, FMT, DP, NR, true> : k_weigh_step<false, FMT, DP, NR, true>)
                : (bf16 ? k_weigh_step<true, FMT, DP, NR, false> : k_weigh_step<false, FMT, DP, NR, false>);
}
template <int FMT>
Kernel pick_dim(bool bf16, int D, bool few, bool even) {
    return D <= 64 ? (few ? pick_even<FMT, 64, 1>(bf16, even) : pick_even<FMT, 64, 2>(bf16, even))
                   : (few ? pick_even<FMT, 128, 1>(bf16, even) : pick_even<FMT, 128, 2>(bf16, even));
}

}  // namespace

cudaError_t launch_weigh_step(const WeighLaunch &a, bool bf16, int fmt, int rows, int sms, cudaStream_t st) {
    const bool few = rows <= 8, even = a.a.c.b % 16 == 0;
    const Kernel k = fmt == kFmt16 ? pick_dim<kFmt16>(bf16, a.a.c.D, few, even)
                   : fmt == kFmtE4M3 ? pick_dim<kFmtE4M3>(bf16, a.a.c.D, few, even)
                                     : pick_dim<kFmtInt8>(bf16, a.a.c.D, few, even);
    return launch_chained(k, (few && fmt == kFmt16 ? 5 : 4) * sms, kThreads, 0, st, a);
}

// Sequences of up to 8 rows (new tokens x query heads of a KV head), or up to 16 if a batch has no more, are the step
// kernel's, others the chunk kernel's.  A single sequence, and as many tokens as if all sequences brought the most, take one launch (the
// other is 5 us with nothing to do).
cudaError_t launch_weigh(const WeighLaunch &a, const CacheMaps &m, bool bf16, int fmt, int sms, cudaStream_t st) {
    const long long most = (long long)a.a.b.max_q * a.a.c.G;
    const int few = most <= 16 || a.a.c.G > 8 ? 16 : 8;
    WeighLaunch l = a;
    if (most > few) {
        const bool all = a.a.b.n == 1 || (long long)a.a.b.n * a.a.b.max_q <= a.a.b.T;
        l.a.row_lo = all ? 1 : few + 1;
        l.a.row_hi = 0x7fffffff;
        const cudaError_t e = launch_weigh_chunk(l, m, bf16, fmt, sms, st);
        if (e != cudaSuccess || all || a.a.c.G > few) return e;
    }
    l.a.row_lo = 1;
    l.a.row_hi = (int)std::min<long long>(most, few);
    return launch_weigh_step(l, bf16, fmt, l.a.row_hi, sms, st);
}

}  // namespace lr
