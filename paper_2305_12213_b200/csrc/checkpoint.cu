// Activation checkpoints in 8 bits as calls of their own (the layers' forward passes write the same format themselves).
#include <algorithm>
#include <cstring>

#include "common.h"
#include "layer_gemm.cuh"

namespace dynbatch {
namespace {

using bf16 = __nv_bfloat16;

// HBM-bound: 3 + 1/32 bytes a value.  A thread has 8 values of a row, four neighbouring threads a group of 32, whose
// maximum they find with two exchanges (16384 x 2048: 18.6 us, 5.5 TB/s, issue slots 74 % busy); a power-of-two number of threads takes a row (blockIdx.y counts the parts of rows
// wider than 2048) and each thread four rows at once, so that four 16-byte loads are under way.  No division and no loop.
constexpr int kBlock = 256, kRowsAtOnce = 4;

struct PackArgs {
    const bf16* x; long long x_pitch;
    uint8_t* codes; uint8_t* scale;
    long long rows;
    int cols, groups, threads_shift;
};

__global__ void __launch_bounds__(kBlock) checkpoint_pack_kernel(const __grid_constant__ PackArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int shift = a.threads_shift, row_groups = kBlock >> shift;
    const int piece = (blockIdx.y << shift) + (threadIdx.x & ((1 << shift) - 1)), col = piece * 8;
    const int n = max(0, min(8, a.cols - col));
    const long long first = static_cast<long long>(blockIdx.x) * (kRowsAtOnce * row_groups) + (threadIdx.x >> shift);
    lg::Raw8<bf16> raw[kRowsAtOnce];
#pragma unroll
    for (int d = 0; d < kRowsAtOnce; ++d) {
        const long long row = first + d * row_groups;
        raw[d].load(a.x + row * a.x_pitch + col, row < a.rows ? n : 0);
    }
#pragma unroll
    for (int d = 0; d < kRowsAtOnce; ++d) {
        const long long row = first + d * row_groups;
        float v[8];
        raw[d].values(v);
        float top = 0.f;                                             // maxima pass NaN over
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));      // whole warps are here
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        uint32_t byte = ck8::scale_byte(top), c0, c1;
        const bool plain = byte < ck8::kTopByte;
        if (!__all_sync(0xFFFFFFFFu, plain)) {                       // infinities, or values near the largest
            float finite = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) finite = fmaxf(finite, ck8::finite_magnitude(v[j]));
            finite = fmaxf(finite, __shfl_xor_sync(0xFFFFFFFFu, finite, 1));
            finite = fmaxf(finite, __shfl_xor_sync(0xFFFFFFFFu, finite, 2));
            byte = ck8::scale_byte(finite);
        }
        if (row < a.rows && n > 0) {
            const float inverse = ck8::scale_inverse(byte);
            if (plain) {
                c0 = ck8::codes_of_finite(v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse);
                c1 = ck8::codes_of_finite(v[4] * inverse, v[5] * inverse, v[6] * inverse, v[7] * inverse);
            } else {
                c0 = ck8::codes4(v[0], v[1], v[2], v[3], inverse, byte);
                c1 = ck8::codes4(v[4], v[5], v[6], v[7], inverse, byte);
            }
            if ((piece & 3) == 0) a.scale[row * a.groups + piece / 4] = static_cast<uint8_t>(byte);
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
}

struct UnpackArgs {
    const uint8_t* codes; const uint8_t* scale;
    bf16* x; long long x_pitch;
    long long rows;
    int cols, groups, threads_shift;
};

__global__ void __launch_bounds__(kBlock) checkpoint_unpack_kernel(const __grid_constant__ UnpackArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int shift = a.threads_shift, row_groups = kBlock >> shift;
    const int col = ((blockIdx.y << shift) + (threadIdx.x & ((1 << shift) - 1))) * 8, n = min(8, a.cols - col);
    if (n <= 0) return;
    const long long first = static_cast<long long>(blockIdx.x) * (kRowsAtOnce * row_groups) + (threadIdx.x >> shift);
    lg::Codes8 c[kRowsAtOnce];
    uint32_t byte[kRowsAtOnce];
#pragma unroll
    for (int d = 0; d < kRowsAtOnce; ++d) {
        const long long row = first + d * row_groups;
        byte[d] = row < a.rows ? a.scale[row * a.groups + col / ck8::kGroup] : 0;
        c[d].load(a.codes + row * a.cols + col, row < a.rows ? n : 0);
    }
#pragma unroll
    for (int d = 0; d < kRowsAtOnce; ++d) {
        const long long row = first + d * row_groups;
        if (row >= a.rows) break;
        lg::Pair v[4];
        c[d].values(byte[d], v);
        bf16* to = a.x + row * a.x_pitch + col;
        if (n == 8 && lg::aligned_to(to, 16)) {
            *reinterpret_cast<uint4*>(to) = make_uint4(lg::pack_pair(v[0]), lg::pack_pair(v[1]), lg::pack_pair(v[2]), lg::pack_pair(v[3]));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x, y;
                lg::halves(v[j], x, y);
                if (2 * j < n) to[2 * j] = __float2bfloat16_rn(x);
                if (2 * j + 1 < n) to[2 * j + 1] = __float2bfloat16_rn(y);
            }
        }
    }
}

bool valid(long long rows, long long cols) { return rows >= 0 && rows <= (1LL << 38) && cols >= 1 && cols <= (1LL << 24) && rows * cols <= (1LL << 40); }

// Threads that take a row: a power of two from four (a group of 32 values) to a CTA's.
int shift_of(long long cols) {
    int s = 2;
    while ((1 << s) < kBlock && (8LL << s) < cols) ++s;
    return s;
}

template <class Args>
db_status launch(void (*fn)(const Args), const Args& a, cudaStream_t stream) {
    const long long per_cta = static_cast<long long>(kRowsAtOnce) * (kBlock >> a.threads_shift), across = 8LL << a.threads_shift;
    const long long ctas = (a.rows + per_cta - 1) / per_cta;
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(static_cast<unsigned>(ctas), static_cast<unsigned>((a.cols + across - 1) / across));
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
    const PackArgs a{static_cast<const bf16*>(x), x_pitch, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scale), rows, cols, groups, shift_of(cols)};
    return launch(checkpoint_pack_kernel, a, static_cast<cudaStream_t>(cuda_stream));
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
    const UnpackArgs a{static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scale), static_cast<bf16*>(x), x_pitch, rows, cols, groups, shift_of(cols)};
    return launch(checkpoint_unpack_kernel, a, static_cast<cudaStream_t>(cuda_stream));
}
