// cuTensorMapEncodeTiled, looked up through the runtime so that the library needs no link against the driver.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "common.h"

namespace dynbatch {

struct TensorMapSpec {
    CUtensorMapDataType type;
    int rank;                           // at most 3; the innermost dimension first
    const void* base;
    cuuint64_t dims[3], strides[2];     // strides in bytes, of the dimensions behind the innermost
    cuuint32_t box[3];
    CUtensorMapSwizzle swizzle;
    CUtensorMapL2promotion l2;
};

// Elements outside the dimensions read as zero.  `rejected`: the message where the driver does not take the layout.
inline db_status encode_tensor_map(CUtensorMap* map, const TensorMapSpec& s, const char* rejected) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<Encode>(p);
    }();
    if (!encode) {
        record_message("cuTensorMapEncodeTiled is not available from this driver");
        return DB_ERR_CUDA;
    }
    const cuuint32_t each[3] = {1, 1, 1};
    const auto call = [&] {
        return encode(map, s.type, static_cast<cuuint32_t>(s.rank), const_cast<void*>(s.base), s.dims, s.strides, s.box, each,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, s.swizzle, s.l2, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = call();
    if (r != CUDA_SUCCESS) {
        // a host thread that has not yet called the runtime for its device has no context, which the driver's call needs
        int device = 0;
        DB_CUDA_TRY(cudaGetDevice(&device));
        DB_CUDA_TRY(cudaSetDevice(device));
        r = call();
    }
    if (r != CUDA_SUCCESS) {
        record_message(rejected);
        return DB_ERR_CUDA;
    }
    return DB_OK;
}

}  // namespace dynbatch
