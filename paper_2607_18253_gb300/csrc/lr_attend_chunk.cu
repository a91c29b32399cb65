// Attention of many rows over a paged KV cache: the kernels of causal batches, the tensor maps, and the calls of all
// (lr_attend_chunk.cuh).
#include "lr_attend_chunk.cuh"

namespace lr {

namespace {

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                            const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {  // the driver's function, looked up once; null if it has none
    static const Encode fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return (Encode) nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    return fn;
}
// A map of 16-bit elements: 64 of the first dimension a box, zeros beyond the tensor, rows of 128 bytes swizzled.
bool encode(CUtensorMap &map, bool bf16, int dims, const void *at, const cuuint64_t *size, const cuuint64_t *stride, const cuuint32_t *box) {
    const cuuint32_t steps[4] = {1, 1, 1, 1};
    for (int i = 0; i + 1 < dims; ++i)
        if (stride[i] == 0 || stride[i] >= (1ull << 40)) return false;
    return encoder() && encoder()(&map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)dims,
                                  const_cast<void *>(at), size, stride, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

int encode_maps(const CacheDev &c, bool bf16, CacheMaps &m) {
    m.box = 0;
    const int box = c.b & -c.b;  // the largest power of two in a block
    if (box < 8) return 0;
    const cuuint32_t tokens = (cuuint32_t)(box < kTok ? box : kTok);
    const cuuint64_t dims[4] = {(cuuint64_t)c.D, (cuuint64_t)c.b, (cuuint64_t)c.H, (cuuint64_t)c.nb};
    // (the stride of a dimension of one element is never used, but has to be one)
    const cuuint64_t strides[3] = {(cuuint64_t)(c.b > 1 ? c.st : 256), (cuuint64_t)(c.H > 1 ? c.sh : 256), (cuuint64_t)(c.nb > 1 ? c.sb : 256)};
    const cuuint32_t boxes[4] = {64, tokens, 1, 1};
    for (int y = 0; y < 2; ++y)
        if (!encode(y ? m.v : m.k, bf16, 4, y ? c.v : c.k, dims, strides, boxes)) return 0;
    return m.box = (int)tokens;
}

bool encode_rows(const AttendLaunch &a, bool bf16, CUtensorMap &map) {
    const CacheDev &c = a.c;
    if (c.G > 128) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)c.D, (cuuint64_t)c.Hq, (cuuint64_t)a.b.T};
    const cuuint64_t strides[2] = {(cuuint64_t)(c.Hq > 1 ? a.q_h : 256), (cuuint64_t)(a.b.T > 1 ? a.q_t : 256)};
    const cuuint32_t box[3] = {64, (cuuint32_t)c.G, (cuuint32_t)(128 / c.G)};
    return encode(map, bf16, 3, a.q, dims, strides, box);
}

cudaError_t attend_chunk_init() {
    cudaError_t e = chunk_init<false>();
    if (e == cudaSuccess) e = tree_chunk_init();
    if (e == cudaSuccess) e = weigh_init();
    if (e == cudaSuccess) e = select_init();
    if (e == cudaSuccess) e = keep_init();
    return e;
}

cudaError_t launch_attend_chunk(const AttendLaunch &a, const CacheMaps &m, bool bf16, int fmt, int ctas, cudaStream_t st) {
    return a.tree ? launch_tree_chunk(a, m, bf16, fmt, ctas, st) : launch_chunk<false>(a, m, bf16, fmt, ctas, st);
}

}  // namespace lr
