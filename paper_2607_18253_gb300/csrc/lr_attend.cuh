// What the attention kernels share: which cached tokens a tile of rows sees, the walk over a
// batch's tiles, conversions of 8-bit codes, and the small PTX wrappers.
#pragma once

#include "lr_cache.cuh"

namespace lr {

// A unit: one sequence, one KV head and one tile of rows.  A row is a (new token, query head of
// the KV head) pair, token-major, so that the query heads that share a KV head share its
// tiles of cached tokens.  The cached tokens that some row of the unit sees are at most two ranges, the sinks
// and the window; they are taken in tiles of TILE tokens.
struct Unit {
    int s, h, qt;      // sequence, KV head, tile of rows
    int q0, ql, kv;    // first row of the token arrays, new tokens, tokens
    int ns, wf, nt;    // tiles of sinks before the window, the window's first tile, tiles in all
    int lo, hi;        // positions of the first and last row
    int rows;          // rows of this tile
};

template <int TILE>
__device__ __forceinline__ int tile_count(int lo, int hi, int window, int sinks, int &ns, int &wf) {
    ns = wf = 0;
    if (hi < 0) return 1;  // nothing to see: one tile, all masked, writes the zeros
    if (window > 0) {
        const int first = max(0, lo - window + 1);
        wf = first / TILE;
        ns = (min(sinks, first) + TILE - 1) / TILE;
        if (ns >= wf) ns = wf = 0;  // the sinks reach the window's first tile
    }
    return ns + hi / TILE - wf + 1;
}

// Sequence s as the batch gives it, false if it is not this launch's: no rows, a number of rows
// outside [row_lo, row_hi], or values out of range (recorded).
__device__ __forceinline__ bool load_seq(const AttendLaunch &a, int s, int &q0, int &ql, int &kv) {
    q0 = __ldg(a.b.q_start + s);
    ql = __ldg(a.b.q_start + s + 1) - q0;
    kv = __ldg(a.b.kv_len + s);
    if (ql == 0) return false;
    if (q0 < 0 || ql < 0 || ql > a.b.max_q || ql > a.b.T - q0 || kv < 0 || kv > kMaxTokens ||
        (long long)kv > (long long)a.b.max_blocks * a.c.b) {
        report(a.c.status, kEInval);
        return false;
    }
    const int rows = ql * a.c.G;
    return rows >= a.row_lo && rows <= a.row_hi;
}

template <int ROWS, int TILE>
__device__ __forceinline__ void set_tile(const AttendLaunch &a, Unit &u) {
    const int r0 = u.qt * ROWS;
    u.rows = min(ROWS, u.ql * a.c.G - r0);
    u.lo = u.kv - u.ql + quot(r0, a.c.div_g);
    u.hi = u.kv - u.ql + quot(r0 + u.rows - 1, a.c.div_g);
    u.nt = tile_count<TILE>(u.lo, u.hi, a.window, a.sinks, u.ns, u.wf);
}

// Tiles of a sequence for one KV head, with the units' weights, a warp's lanes taking its tiles of rows in
// turn (all call).
template <int ROWS, int TILE, int WEIGHT>
__device__ __forceinline__ long long seq_tiles(const AttendLaunch &a, int s) {
    Unit u;
    u.s = s;
    if (!load_seq(a, s, u.q0, u.ql, u.kv)) return 0;
    const int nq = (u.ql * a.c.G + ROWS - 1) / ROWS;
    long long n = 0;
    for (u.qt = threadIdx.x & 31; u.qt < nq; u.qt += 32) {
        set_tile<ROWS, TILE>(a, u);
        n += u.nt + WEIGHT;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    return n;
}

// The batch's tiles in one line, units in order of sequence, KV head, tile of rows, cut into equal shares for the
// CTAs.  A unit counts WEIGHT more than its tiles, at its front, for what it costs to begin and end one: a cut
// that falls there takes the unit whole.
struct Share {
    long long x0, x1, all;  // this CTA's share, of the whole
    int ctas;               // by so many CTAs (the others have none)
};

// A position in the line, within a CTA's share.
template <int ROWS, int TILE, int WEIGHT>
struct Cursor {
    Unit u;
    int j, end;    // tile of the unit; the CTA's tiles of it end there
    bool last;     // its last unit
    long long at;  // where the unit begins
    __device__ __forceinline__ int base() const { return (j < u.ns ? j : u.wf + j - u.ns) * TILE; }
    __device__ __forceinline__ bool more() const { return j + 1 < end || !last; }
    __device__ __forceinline__ bool whole() const { return j == 0 && end == u.nt; }  // (at the unit's first tile)
    __device__ __forceinline__ void enter(const AttendLaunch &a, const Share &s) {
        set_tile<ROWS, TILE>(a, u);
        end = (int)min((long long)u.nt, s.x1 - at - WEIGHT);
        last = at + u.nt + 2 * WEIGHT >= s.x1;
    }
    __device__ __forceinline__ void next(const AttendLaunch &a, const Share &s) {  // there is more
        if (++j < end) return;
        j = 0;
        at += u.nt + WEIGHT;
        if ((++u.qt) * ROWS >= u.ql * a.c.G) {
            u.qt = 0;
            if (++u.h == a.c.H) {
                u.h = 0;
                do ++u.s;
                while (u.s < a.b.n && !load_seq(a, u.s, u.q0, u.ql, u.kv));
            }
        }
        enter(a, s);
    }
};

// Inclusive sum over a CTA of THREADS threads (all take part); `total` is the sum of all.
template <int THREADS>
__device__ __forceinline__ long long block_sum(long long v, long long *sh, long long &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    __syncthreads();
    if (lane == 31) sh[w] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < w) v += sh[i];
        total += sh[i];
    }
    return v;
}

// The start of CTA c's share (32-bit divisions where they do, as nearly always).
__device__ __forceinline__ long long share_start(const Share &s, int c) {
    return s.all < 1 << 20 ? (long long)((uint32_t)s.all * (uint32_t)c / (uint32_t)s.ctas) : s.all * c / s.ctas;
}
// (scratch: THREADS / 32 + 2 words of shared memory)
// This CTA's share, LEAST or more long, with `cur` at its first tile; false if it has none.
template <int ROWS, int TILE, int WEIGHT, int THREADS, int LEAST>
__device__ __forceinline__ bool take_share(const AttendLaunch &a, Cursor<ROWS, TILE, WEIGHT> &cur, Share &sh, long long *scratch) {
    long long *const s_sum = scratch, &s_rest = scratch[THREADS / 32], &s_seq = scratch[THREADS / 32 + 1];
    const int n = a.b.n, tid = threadIdx.x, lane = tid & 31;
    // tiles of sequence base + tid: a thread's own look where no sequence has more than one tile of rows,
    // else a warp together for each of its threads
    const bool single = (long long)a.b.max_q * a.c.G <= ROWS;
    auto tiles_of = [&](int base) -> long long {
        if (single) {
            Unit u;
            u.s = base + tid;
            u.qt = 0;
            if (u.s >= n || !load_seq(a, u.s, u.q0, u.ql, u.kv)) return 0;
            set_tile<ROWS, TILE>(a, u);
            return (long long)a.c.H * (u.nt + WEIGHT);
        }
        long long mine = 0;
        const int w0 = base + tid - lane;
        for (int i = 0; i < 32 && w0 + i < n; ++i) {
            const long long t = a.c.H * seq_tiles<ROWS, TILE, WEIGHT>(a, w0 + i);
            if (i == lane) mine = t;
        }
        return mine;
    };
    long long all = 0, first = 0, incl = 0, mine = 0;
    for (int base = 0; base < n; base += THREADS) {
        mine = tiles_of(base);
        long long t;
        incl = block_sum<THREADS>(mine, s_sum, t);
        all += t;
    }
    if (all == 0) return false;
    sh.all = all;
    sh.ctas = (int)min((long long)gridDim.x, max(all / LEAST, 1ll));
    const int c = blockIdx.x;
    if (c >= sh.ctas) return false;
    sh.x0 = share_start(sh, c);
    sh.x1 = share_start(sh, c + 1);
    for (int base = 0; base < n; base += THREADS) {
        long long t;
        if (n > THREADS) {
            mine = tiles_of(base);
            incl = block_sum<THREADS>(mine, s_sum, t);
        } else {
            t = all;
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
    Unit &u = cur.u;
    u.s = (int)s_seq;
    load_seq(a, u.s, u.q0, u.ql, u.kv);
    long long r = s_rest;
    const long long per = seq_tiles<ROWS, TILE, WEIGHT>(a, u.s);
    u.h = (int)(r / per);
    r -= u.h * per;
    const int nq = (u.ql * a.c.G + ROWS - 1) / ROWS;
    for (int q0 = 0;; q0 += 32) {  // 32 tiles of rows at a time
        u.qt = min(q0 + lane, nq - 1);
        set_tile<ROWS, TILE>(a, u);
        const long long own = q0 + lane < nq ? u.nt + WEIGHT : 0;
        long long upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, r < upto);
        if (hit) {
            const int at = __ffs(hit) - 1;
            r -= __shfl_sync(0xffffffffu, upto - own, at);
            u.qt = q0 + at;
            break;
        }
        r -= __shfl_sync(0xffffffffu, upto, 31);
    }
    cur.at = sh.x0 - r;
    cur.enter(a, sh);
    cur.j = max(0, (int)r - WEIGHT);
    return cur.j < cur.end;  // (a share may end in a unit's weight)
}

// The CTA that has position x, and where CTA c's part of the unit that begins at `at` lies: its first unit in slot
// 2c, a later one in slot 2c + 1.
__device__ __forceinline__ int cta_of(const Share &s, long long x) {
    return s.all < 1 << 20 ? (int)((((uint32_t)x + 1) * (uint32_t)s.ctas - 1) / (uint32_t)s.all) : (int)(((x + 1) * s.ctas - 1) / s.all);
}
__device__ __forceinline__ int slot_of(const Share &s, int c, long long at) { return 2 * c + (share_start(s, c) < at ? 1 : 0); }

__device__ __forceinline__ bool visible(int pos, int j, int window, int sinks) {
    return j <= pos && (window == 0 || j > pos - window || j < sinks);
}

// Bytes i and j of w, 8-bit codes, as two bf16 numbers (i in the low half), exactly.  e4m3: sign, four exponent
// and three mantissa bits moved to their places, then a product with 2^120, the power of two between the
// biases (subnormal codes are subnormal bf16 numbers first, which the product turns right as well).
// int8: 128 + the low seven bits, less 128 or, for a negative code, 256.
template <int FMT>
__device__ __forceinline__ uint32_t to_bf16(uint32_t w, int i, int j) {
    uint32_t d;
    if constexpr (FMT == kFmtE4M3) {
        const uint32_t t = __byte_perm(w, 0, 0x0404u | i << 4 | j << 12);
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"((t & 0x80008000u) | ((t >> 4) & 0x07f007f0u)), "r"(0x7b807b80u));
    } else {
        const uint32_t t = __byte_perm(w, 0, 0x4040u | i | j << 8);
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"((t & 0x007f007fu) | 0x43004300u), "r"((t & 0x00800080u) | 0x43004300u));
    }
    return d;
}
// Four 8-bit codes to fp16 numbers, exactly, as two pairs: codes (0, 1) and (2, 3), or with SPLIT (0, 2) and
// (1, 3).  e4m3 by the conversion instruction.  int8: 1024 + (code + 128), less 1152.
template <int FMT, bool SPLIT>
__device__ __forceinline__ void to_half(uint32_t w, uint32_t &a, uint32_t &b) {
    if constexpr (FMT == kFmtE4M3) {
        if constexpr (SPLIT) w = __byte_perm(w, 0, 0x3120);
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(a), "=r"(b) : "r"(w));
    } else {
        w ^= 0x80808080u;
        a = __byte_perm(w, 0x64646464u, SPLIT ? 0x4240 : 0x4140);
        b = __byte_perm(w, 0x64646464u, SPLIT ? 0x4341 : 0x4342);
        asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(a) : "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(b) : "r"(0x64806480u));
    }
}
// e4m3's codes for NaN set to zero.
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
    const uint32_t x = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // the high bit of each such byte
    return w & ~(x | (x - (x >> 7)));
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool BF16>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
    if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<__half2 *>(&x));
}
// An infinity or a NaN among the two 16-bit numbers.
template <bool BF16>
__device__ __forceinline__ bool not_finite(uint32_t x) {
    constexpr uint32_t e = BF16 ? 0x7f80u : 0x7c00u;
    return (x & e) == e || (x >> 16 & e) == e;
}

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes of global memory to shared memory, zeros if `ok` is false.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

}  // namespace lr
