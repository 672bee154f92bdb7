// tensor_map.cu -- tensor maps for the bulk tensor copies: the driver's
// encoder, found once, and the shapes that the operators use.
#include "tensor_map.cuh"

#include "attention.cuh"

namespace sieve {
namespace enc {

sieve_status encode_map(CUtensorMap *map, CUtensorMapDataType type, int rank, const void *base, const cuuint64_t *dims,
                        const cuuint64_t *strides, const cuuint32_t *box) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    // the driver's function, found once (the first caller's thread looks, the
    // others wait for it)
    struct Found {
        Encode fn = nullptr;
        cudaError_t error;
        Found() {
            void *p = nullptr;
            cudaDriverEntryPointQueryResult how = cudaDriverEntryPointSymbolNotFound;
            error = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how);
            if (error == cudaSuccess && how == cudaDriverEntryPointSuccess) fn = reinterpret_cast<Encode>(p);
        }
    };
    static const Found found;
    if (found.error != cudaSuccess) return record_cuda_error(found.error);
    if (!found.fn) return SIEVE_EUNSUPPORTED;
    const cuuint32_t step[3] = {1, 1, 1};
    auto make = [&] {
        return found.fn(map, type, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, step,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = make();
    if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
        // The driver's functions want a current context, and a host thread has
        // none before its first call of the runtime that needs one.
        int dev;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaSetDevice(dev);
        if (e != cudaSuccess) return record_cuda_error(e);
        r = make();
    }
    if (r == CUDA_SUCCESS) return SIEVE_OK;
    return r == CUDA_ERROR_INVALID_VALUE ? SIEVE_EINVAL : record_cuda_error(static_cast<cudaError_t>(r));
}

sieve_status make_map(CUtensorMap *map, int dtype, const void *base, int head_dim, int heads, int64_t tokens,
                      int64_t token_stride, int64_t head_stride, int box_heads, int box_tokens) {
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    // an axis of one element has no stride that matters
    const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? head_stride : head_dim) * 2,
                                   (cuuint64_t)(tokens > 1 ? token_stride : (int64_t)heads * head_dim) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
    return encode_map(map, dtype == SIEVE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                      base, dims, strides, box);
}

sieve_status make_matrix_map(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t width,
                             int64_t stride, int box_rows) {
    const int size = dtype == SIEVE_F32 ? 4 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? stride : width) * size};
    const cuuint32_t box[2] = {128u / size, (cuuint32_t)box_rows};
    return encode_map(map, dtype == SIEVE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                           : dtype == SIEVE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                      2, base, dims, strides, box);
}

}  // namespace enc
}  // namespace sieve
