// Activation checkpoints in 8 bits as calls of their own (the layers' forward passes write the same format themselves).
#include <algorithm>
#include <cstring>

#include "common.h"
#include "layer_gemm.cuh"

namespace dynbatch {
namespace {

using bf16 = __nv_bfloat16;

// HBM-bound: 3 + 1/32 bytes a value.  A thread has 8 values of a row, four neighbouring threads a group of 32, whose
// maximum they find with two exchanges; 16-byte loads and 8-byte stores, whole lines for a warp.
constexpr int kBlock = 256;

struct PackArgs {
    const bf16* x; long long x_pitch;
    uint8_t* codes; uint8_t* scale;
    long long rows;
    int cols, groups;
};

__global__ void __launch_bounds__(kBlock) checkpoint_pack_kernel(const __grid_constant__ PackArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const long long per_row = 4LL * a.groups, total = a.rows * per_row;
    const long long stride = static_cast<long long>(gridDim.x) * kBlock;
    // whole warps stay in the loop: the exchange needs all four threads of a group (a row has a multiple of four)
    for (long long i = static_cast<long long>(blockIdx.x) * kBlock + threadIdx.x; (i & ~31LL) < total; i += stride) {
        const bool in = i < total;
        const long long row = in ? i / per_row : 0;
        const int piece = in ? static_cast<int>(i - row * per_row) : 0, col = piece * 8;
        const int n = in ? max(0, min(8, a.cols - col)) : 0;
        float v[8];
        const bf16* p = a.x + row * a.x_pitch + col;
        if (n == 8 && lg::aligned_to(p, 16)) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            lg::unpack2(q.x, v[0], v[1]); lg::unpack2(q.y, v[2], v[3]);
            lg::unpack2(q.z, v[4], v[5]); lg::unpack2(q.w, v[6], v[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? __bfloat162float(p[j]) : 0.f;
        }
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, ck8::finite_magnitude(v[j]));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        if (!in) continue;
        const uint32_t byte = ck8::scale_byte(top);
        const float inverse = ck8::scale_inverse(byte);
        if ((piece & 3) == 0) a.scale[row * a.groups + piece / 4] = static_cast<uint8_t>(byte);
        const uint32_t c0 = ck8::codes4(v[0], v[1], v[2], v[3], inverse, byte), c1 = ck8::codes4(v[4], v[5], v[6], v[7], inverse, byte);
        uint8_t* to = a.codes + row * a.cols + col;
        if (n == 8 && lg::aligned_to(to, 8)) {
            __stcs(reinterpret_cast<uint2*>(to), make_uint2(c0, c1));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) to[j] = static_cast<uint8_t>((j < 4 ? c0 : c1) >> (8 * (j % 4)));
        }
    }
}

struct UnpackArgs {
    const uint8_t* codes; const uint8_t* scale;
    bf16* x; long long x_pitch;
    long long rows;
    int cols, groups;
};

__global__ void __launch_bounds__(kBlock) checkpoint_unpack_kernel(const __grid_constant__ UnpackArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const long long per_row = (a.cols + 7) / 8, total = a.rows * per_row;
    const long long stride = static_cast<long long>(gridDim.x) * kBlock;
    for (long long i = static_cast<long long>(blockIdx.x) * kBlock + threadIdx.x; i < total; i += stride) {
        const long long row = i / per_row;
        const int col = static_cast<int>(i - row * per_row) * 8, n = min(8, a.cols - col);
        const float scale = ck8::scale_value(a.scale[row * a.groups + col / ck8::kGroup]);
        const uint8_t* p = a.codes + row * a.cols + col;
        uint32_t c[2] = {0, 0};
        if (n == 8 && lg::aligned_to(p, 8)) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            c[0] = q.x; c[1] = q.y;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) c[j / 4] |= static_cast<uint32_t>(p[j]) << (8 * (j % 4));
        }
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float2 t = ck8::values2(c[j / 4] >> (8 * (j % 4)));
            v[j] = t.x * scale; v[j + 1] = t.y * scale;
        }
        bf16* to = a.x + row * a.x_pitch + col;
        if (n == 8 && lg::aligned_to(to, 16)) {
            *reinterpret_cast<uint4*>(to) = make_uint4(lg::pack2(v[0], v[1]), lg::pack2(v[2], v[3]), lg::pack2(v[4], v[5]), lg::pack2(v[6], v[7]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) to[j] = __float2bfloat16_rn(v[j]);
        }
    }
}

bool valid(long long rows, long long cols) { return rows >= 0 && rows <= (1LL << 40) && cols >= 1 && cols <= (1LL << 24) && rows * cols <= (1LL << 40); }

template <class Args>
db_status launch(void (*fn)(const Args), const Args& a, long long pieces, cudaStream_t stream) {
    // eight CTAs of 256 threads fill an SM
    const long long ctas = std::min<long long>((pieces + kBlock - 1) / kBlock, 8LL * sm_count());
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(kBlock);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    DB_CUDA_TRY(cudaLaunchKernelEx(&cfg, fn, a));
    return DB_OK;
}

bool apart(const void* a, long long na, const void* b, long long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na <= 0 || nb <= 0 || x + static_cast<uintptr_t>(na) <= y || y + static_cast<uintptr_t>(nb) <= x;
}

}  // namespace
}  // namespace dynbatch

extern "C" db_status db_checkpoint_pack(const void* x, int64_t x_pitch, int64_t rows, int32_t cols, void* codes, void* scale,
                                        void* cuda_stream) {
    using namespace dynbatch;
    if (!valid(rows, cols)) return DB_ERR_ARG;
    if (rows == 0) return DB_OK;
    if (!x || !codes || !scale) return DB_ERR_NULL;
    if (x_pitch < cols || x_pitch > (1LL << 31) || reinterpret_cast<uintptr_t>(x) % 2) return DB_ERR_ARG;
    const int groups = (cols + ck8::kGroup - 1) / ck8::kGroup;
    const long long nx = ((rows - 1) * x_pitch + cols) * 2, nc = rows * cols, ns = rows * groups;
    if (!apart(x, nx, codes, nc) || !apart(x, nx, scale, ns) || !apart(codes, nc, scale, ns)) return DB_ERR_ARG;
    const PackArgs a{static_cast<const bf16*>(x), x_pitch, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scale), rows, cols, groups};
    return launch(checkpoint_pack_kernel, a, rows * 4 * groups, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" db_status db_checkpoint_unpack(const void* codes, const void* scale, int64_t rows, int32_t cols, void* x,
                                          int64_t x_pitch, void* cuda_stream) {
    using namespace dynbatch;
    if (!valid(rows, cols)) return DB_ERR_ARG;
    if (rows == 0) return DB_OK;
    if (!x || !codes || !scale) return DB_ERR_NULL;
    if (x_pitch < cols || x_pitch > (1LL << 31) || reinterpret_cast<uintptr_t>(x) % 2) return DB_ERR_ARG;
    const int groups = (cols + ck8::kGroup - 1) / ck8::kGroup;
    const long long nx = ((rows - 1) * x_pitch + cols) * 2, nc = rows * cols, ns = rows * groups;
    if (!apart(x, nx, codes, nc) || !apart(x, nx, scale, ns)) return DB_ERR_ARG;
    const UnpackArgs a{static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scale), static_cast<bf16*>(x), x_pitch, rows, cols, groups};
    return launch(checkpoint_unpack_kernel, a, rows * ((cols + 7) / 8), static_cast<cudaStream_t>(cuda_stream));
}
