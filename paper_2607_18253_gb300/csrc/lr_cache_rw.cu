// Store and load of a paged KV cache: new K and V converted to the cache's format as they are
// written to their blocks, and cached vectors read back as values.
//
// Sixteen lanes hold one vector, eight elements each (the largest magnitude of a vector
// is four shuffles); a CTA takes 64 consecutive (token, head) pairs, four a group of lanes with
// their loads issued together, K and V of a pair by the same lanes; as it stores 8 bits, 32 pairs, two a group.  The CTA's tokens are looked up once
// (sequence, then block table) and kept in shared memory.
#include <cuda_fp8.h>

#include "lr_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256, kGroups = kThreads / 16;
// (token, head) pairs a group of lanes: four where their bytes are only moved (6.9 TB/s), two where they are
// converted as they are stored, which takes registers (8,192 tokens of 8 heads to int8: 30 and 17 us, of which the
// bytes are 7.5: 2,048 CTAs are 3.4 waves, each a chain of lookups, vectors and conversion)
template <int FMT>
constexpr int kStoreItems = FMT == kFmt16 ? 4 : 2;
constexpr int kLoadItems = 4, kMostTokens = kGroups * 4 + 1;

struct Place {
    int64_t off;  // byte offset of the token's place for head 0, -1: none, -2: of no sequence
    int64_t soff; // the same in the scales
};

// The place of token t, which is token t - begin of sequence s's [begin, end).
__device__ __forceinline__ Place find_place(const CacheDev &c, const BatchDev &b, int s, int end, int t) {
    Place p{-1, 0};
    const int kv = __ldg(b.kv_len + s), pos = kv - (end - t);
    if (pos < 0 || kv > kMaxTokens) return p;
    int place;
    const int64_t blk = block_of(c, b, s, pos, place);
    if (blk < 0) return p;
    p.off = blk * c.sb + place * c.st;
    p.soff = blk * c.ssb + place * c.sst;
    return p;
}

// The places of the CTA's tokens t0 .. t1 - 1 (at most kMostTokens of them), in shared memory.  The sequences that have
// them are found by all threads together, a sequence each: one round of loads for 256 sequences, where a
// search takes one a halving (64 tokens of 64 sequences stored and read back: 8.6 us, searched for
// 9.5).  More than kScan sequences are searched for.
// Where q_start is out of order several sequences may claim a token, which then has no place: the scan finds
// that out, and each token counts its claims.  (A search does not: its token goes to one of them; the launch's CTAs look
// through the order together.)
constexpr int kScan = 1024;
__device__ __noinline__ int2 only_claim(const BatchDev &b, int t) {
    int2 e = make_int2(-1, 0);
    for (int s = 0; s < b.n; ++s) {
        const int end = __ldg(b.q_start + s + 1);
        if (__ldg(b.q_start + s) > t || t >= end) continue;
        if (e.x >= 0) return make_int2(-2, 0);
        e = make_int2(s, end);
    }
    return e;
}
__device__ __forceinline__ void find_places(Place *sp, int2 *seq, const CacheDev &c, const BatchDev &b, int t0, int t1) {
    const int mine = t0 + (int)threadIdx.x;
    if (mine < t1) seq[threadIdx.x] = make_int2(-1, 0);
    bool disorder = false;
    __syncthreads();
    if (b.n <= kScan) {
        for (int s = threadIdx.x; s < b.n; s += kThreads) {
            const int begin = __ldg(b.q_start + s), end = __ldg(b.q_start + s + 1);
            if (begin > end) {
                report(c.status, kEInval);
                disorder = true;
            }
            for (int t = max(begin, t0); t < min(end, t1); ++t) seq[t - t0] = make_int2(s, end);
        }
    } else {
        for (int64_t s = (int64_t)blockIdx.x * kThreads + threadIdx.x; s < b.n; s += (int64_t)gridDim.x * kThreads)
            if (__ldg(b.q_start + s) > __ldg(b.q_start + s + 1)) report(c.status, kEInval);
        // the last sequence that begins at or before the token
        int lo = 0, hi = mine < t1 ? b.n : 0;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(b.q_start + mid) <= mine) lo = mid + 1;
            else hi = mid;
        }
        if (lo > 0) {
            const int end = __ldg(b.q_start + lo);
            if (mine < end) seq[threadIdx.x] = make_int2(lo - 1, end);
            else if (lo < b.n) report(c.status, kEInval);
        }
    }
    disorder = __syncthreads_or(disorder);
    if (mine < t1) {
        const int2 e = disorder ? only_claim(b, mine) : seq[threadIdx.x];
        Place p{e.x == -1 ? -2 : -1, 0};
        if (e.x >= 0) p = find_place(c, b, e.x, e.y, mine);
        if (p.off == -1) report(c.status, kEInval);
        sp[threadIdx.x] = p;
    }
    __syncthreads();
}

template <bool BF16>
__device__ __forceinline__ float2 unpack(uint32_t x) {
    if constexpr (BF16) return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&x));
    else return __half22float2(*reinterpret_cast<__half2 *>(&x));
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack(float a, float b) {
    if constexpr (BF16) {
        __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&r);
    } else {
        __half2 r = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&r);
    }
}

// Eight elements of a vector (its other lanes hold the rest) to 8-bit codes; the scale is the
// same in all lanes.  The largest magnitude is taken over the bits, as integers, where a NaN is
// above infinity and infinity above every number.
template <bool BF16, int FMT>
__device__ __forceinline__ uint2 quantise(const uint4 &w, float &scale) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    float f[8];
    uint32_t top = __float_as_uint(0x1p-100f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = unpack<BF16>(u[i]);
        f[2 * i] = x.x;
        f[2 * i + 1] = x.y;
        top = max(top, max(__float_as_uint(x.x) & 0x7fffffffu, __float_as_uint(x.y) & 0x7fffffffu));
    }
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
    constexpr float kTop = FMT == kFmtE4M3 ? 448.0f : 127.0f;
    const float a = __uint_as_float(top), inv = __fdiv_rn(kTop, a);
    scale = __fdiv_rn(a, kTop);
    if (top >= 0x7f800000u) return make_uint2(0, 0);  // the scale says it all
    uint2 r;
    if constexpr (FMT == kFmtE4M3) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            h[i] = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(f[2 * i], inv), __fmul_rn(f[2 * i + 1], inv)),
                                            __NV_SATFINITE, __NV_E4M3);
        r.x = h[0] | h[1] << 16;
        r.y = h[2] | h[3] << 16;
    } else {
        // 1.5 * 2^23 added: the sum's last bit is one, so it is rounded to an integer (ties to even), which its low bits
        // hold.  The products are at most 127 and a rounding.
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(__fadd_rn(__fmul_rn(f[i], inv), 12582912.0f));
        auto four = [&](int i) { return __byte_perm(__byte_perm(q[i], q[i + 1], 0x0040), __byte_perm(q[i + 2], q[i + 3], 0x0040), 0x5410); };
        r.x = four(0);
        r.y = four(4);
    }
    return r;
}

template <bool BF16, int FMT>
__global__ void __launch_bounds__(kThreads) k_cache_write(const __grid_constant__ RwLaunch a) {
    __shared__ Place sp[kMostTokens];
    __shared__ int2 seq[kMostTokens];
    constexpr int kItems = kStoreItems<FMT>, kPairs = kGroups * kItems;
    chain_wait();
    const CacheDev &c = a.c;
    const int64_t first = (int64_t)blockIdx.x * kPairs, total = (int64_t)a.b.T * c.H;
    const int64_t last = min(first + kPairs, total) - 1;
    const int t0 = (int)(first / c.H), t1 = (int)(last / c.H) + 1;
    const int g = threadIdx.x / 16, l = threadIdx.x % 16;
    const bool on = l * 8 < c.D;
    uint4 k[kItems], v[kItems];
    int tok[kItems], head[kItems];
#pragma unroll
    for (int u = 0; u < kItems; ++u) {  // the new vectors do not wait for their places
        const int64_t i = first + u * kGroups + g;
        tok[u] = -1;
        k[u] = v[u] = make_uint4(0, 0, 0, 0);
        if (i > last) continue;
        tok[u] = (int)(i / c.H);
        head[u] = (int)(i - (int64_t)tok[u] * c.H);
        if (!on) continue;
        const int64_t at = tok[u] * a.in_t + head[u] * a.in_h + l * 16;
        k[u] = __ldcs(reinterpret_cast<const uint4 *>(a.k_in + at));
        v[u] = __ldcs(reinterpret_cast<const uint4 *>(a.v_in + at));
    }
    find_places(sp, seq, c, a.b, t0, t1);
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
        const Place p = tok[u] < 0 ? Place{-2, 0} : sp[tok[u] - t0];
        const int64_t at = p.off + (tok[u] < 0 ? 0 : head[u] * c.sh);
        if constexpr (FMT == kFmt16) {
            if (p.off < 0 || !on) continue;
            *reinterpret_cast<uint4 *>(c.k + at + l * 16) = k[u];
            *reinterpret_cast<uint4 *>(c.v + at + l * 16) = v[u];
        } else {
            float sk, sv;  // (every lane takes part in the shuffles)
            const uint2 qk = quantise<BF16, FMT>(k[u], sk), qv = quantise<BF16, FMT>(v[u], sv);
            if (p.off < 0) continue;
            if (on) {
                *reinterpret_cast<uint2 *>(c.k + at + l * 8) = qk;
                *reinterpret_cast<uint2 *>(c.v + at + l * 8) = qv;
            }
            if (l == 0) {
                c.ks[p.soff + head[u] * c.ssh] = sk;
                c.vs[p.soff + head[u] * c.ssh] = sv;
            }
        }
    }
    chain_next();
}

// Eight cached elements as fp32 values; `w` holds 16-bit elements or, in its first half, codes.
template <bool BF16, int FMT>
__device__ __forceinline__ void values(const uint4 &w, float scale, float *f) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (FMT == kFmt16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = unpack<BF16>(u[i]);
            f[2 * i] = x.x;
            f[2 * i + 1] = x.y;
        }
    } else if constexpr (FMT == kFmtE4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u[i / 2] >> (i % 2 * 16)), __NV_E4M3);
            const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&h));
            f[2 * i] = __fmul_rn(x.x, scale);
            f[2 * i + 1] = __fmul_rn(x.y, scale);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __fmul_rn((float)(int8_t)(u[i / 4] >> (i % 4 * 8)), scale);
    }
}

template <bool BF16, int FMT, bool F32>
__global__ void __launch_bounds__(kThreads) k_cache_read(const __grid_constant__ RwLaunch a) {
    __shared__ Place sp[kMostTokens];
    __shared__ int2 seq[kMostTokens];
    constexpr int kItems = kLoadItems, kPairs = kGroups * kItems;
    chain_wait();
    const CacheDev &c = a.c;
    const int64_t first = (int64_t)blockIdx.x * kPairs, total = (int64_t)a.b.T * c.H;
    const int64_t last = min(first + kPairs, total) - 1;
    const int t0 = (int)(first / c.H), t1 = (int)(last / c.H) + 1;
    const int g = threadIdx.x / 16, l = threadIdx.x % 16;
    const bool on = l * 8 < c.D;
    find_places(sp, seq, c, a.b, t0, t1);
    uint4 k[kItems], v[kItems];
    float sk[kItems], sv[kItems];
    bool write[kItems];
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
        const int64_t i = first + u * kGroups + g;
        write[u] = false;
        if (i > last || !on) continue;
        const int tok = (int)(i / c.H), head = (int)(i - (int64_t)tok * c.H);
        const Place p = sp[tok - t0];
        if (p.off == -2) continue;
        write[u] = true;
        sk[u] = sv[u] = __uint_as_float(0x7fffffffu);
        if constexpr (FMT == kFmt16) {
            constexpr uint32_t kNan = 0x7fff7fffu;  // in either 16-bit type
            k[u] = v[u] = make_uint4(kNan, kNan, kNan, kNan);
            if (p.off < 0) continue;
            k[u] = __ldcs(reinterpret_cast<const uint4 *>(c.k + p.off + head * c.sh + l * 16));
            v[u] = __ldcs(reinterpret_cast<const uint4 *>(c.v + p.off + head * c.sh + l * 16));
        } else {
            k[u] = v[u] = make_uint4(0, 0, 0, 0);
            if (p.off < 0) continue;
            const uint2 x = __ldcs(reinterpret_cast<const uint2 *>(c.k + p.off + head * c.sh + l * 8));
            const uint2 y = __ldcs(reinterpret_cast<const uint2 *>(c.v + p.off + head * c.sh + l * 8));
            k[u] = make_uint4(x.x, x.y, 0, 0);
            v[u] = make_uint4(y.x, y.y, 0, 0);
            sk[u] = c.ks[p.soff + head * c.ssh];
            sv[u] = c.vs[p.soff + head * c.ssh];
        }
    }
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
        if (!write[u]) continue;
        const int64_t at = (first + u * kGroups + g) * c.D + l * 8;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const uint4 &w = y ? v[u] : k[u];
            char *out = y ? a.v_out : a.k_out;
            if constexpr (FMT == kFmt16 && !F32) {
                __stcs(reinterpret_cast<uint4 *>(out + at * 2), w);
            } else {
                float f[8];
                values<BF16, FMT>(w, y ? sv[u] : sk[u], f);
                if constexpr (F32) {
                    __stcs(reinterpret_cast<float4 *>(out + at * 4), make_float4(f[0], f[1], f[2], f[3]));
                    __stcs(reinterpret_cast<float4 *>(out + at * 4) + 1, make_float4(f[4], f[5], f[6], f[7]));
                } else {
                    __stcs(reinterpret_cast<uint4 *>(out + at * 2),
                           make_uint4(pack<BF16>(f[0], f[1]), pack<BF16>(f[2], f[3]), pack<BF16>(f[4], f[5]),
                                      pack<BF16>(f[6], f[7])));
                }
            }
        }
    }
    chain_next();
}

int grid_of(const RwLaunch &a, int items) {
    const int pairs = kGroups * items;
    return (int)(((int64_t)a.b.T * a.c.H + pairs - 1) / pairs);
}

}  // namespace

cudaError_t launch_cache_write(const RwLaunch &a, bool bf16, int fmt, cudaStream_t st) {
    auto go = [&](void (*k)(const RwLaunch)) { return launch_chained(k, grid_of(a, fmt == kFmt16 ? kStoreItems<kFmt16> : kStoreItems<kFmtInt8>), kThreads, 0, st, a); };
    switch (fmt) {
        case kFmtE4M3: return go(bf16 ? k_cache_write<true, kFmtE4M3> : k_cache_write<false, kFmtE4M3>);
        case kFmtInt8: return go(bf16 ? k_cache_write<true, kFmtInt8> : k_cache_write<false, kFmtInt8>);
        default: return go(k_cache_write<true, kFmt16>);  // 16 bits are copied, whatever they are
    }
}

cudaError_t launch_cache_read(const RwLaunch &a, bool bf16, int fmt, bool f32, cudaStream_t st) {
    auto go = [&](void (*k)(const RwLaunch)) { return launch_chained(k, grid_of(a, kLoadItems), kThreads, 0, st, a); };
    switch (fmt) {
        case kFmtE4M3:
            return f32 ? go(k_cache_read<true, kFmtE4M3, true>)
                       : go(bf16 ? k_cache_read<true, kFmtE4M3, false> : k_cache_read<false, kFmtE4M3, false>);
        case kFmtInt8:
            return f32 ? go(k_cache_read<true, kFmtInt8, true>)
                       : go(bf16 ? k_cache_read<true, kFmtInt8, false> : k_cache_read<false, kFmtInt8, false>);
        default:
            return f32 ? go(bf16 ? k_cache_read<true, kFmt16, true> : k_cache_read<false, kFmt16, true>)
                       : go(k_cache_read<true, kFmt16, false>);
    }
}

}  // namespace lr
