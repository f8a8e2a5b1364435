// Host side of the matrix products: tensor maps.  See gpga_gemm.cuh.
#include "gpga_gemm.cuh"

namespace gpga {

namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode find_encoder()
{
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
        return nullptr;
    return reinterpret_cast<Encode>(f);
}

}  // namespace

cudaError_t encode_map(CUtensorMap& map, const Operand& o, bool half, int box_rows)
{
    static const Encode encode = find_encoder();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[4] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.batches, (cuuint64_t)o.pieces};
    // the stride of a dimension of one entry is never used, but must be valid
    const cuuint64_t batch = o.batches > 1 ? o.batch * 2 : 16, piece = o.pieces > 1 ? o.piece * 2 : 16;
    const cuuint64_t strides[3] = {o.outer > 1 ? (cuuint64_t)o.ld * 2 : 16, batch, piece};
    const cuuint32_t box[4] = {kTileK, (cuuint32_t)box_rows, 1, 1}, each[4] = {1, 1, 1, 1};
    const CUresult r = encode(&map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(o.base), dims,
                              strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

bool operand_fits(const void* base, int64_t ld, int64_t batch)
{
    return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && ld % 8 == 0 && batch % 8 == 0 && ld > 0 && batch >= 0 && ld < (int64_t(1) << 39) &&
           batch < (int64_t(1) << 39);
}

int sm_count()
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    std::atomic<int>& k = known[dev & 63];
    int n = k.load();
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 2) n = 148;
        k.store(n);
    }
    return n;
}

}  // namespace gpga
