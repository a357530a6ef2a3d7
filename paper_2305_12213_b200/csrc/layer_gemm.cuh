// The bf16 matrix product of the layers (sm_100a, tcgen05), with what follows it done on the accumulator:
//     acc(m, n) = sum_k A(m, k) * B(n, k)          fp32 in tensor memory, operands bf16 by TMA
// Either operand may have the reduction index or the output index as its contiguous one, so that a layer's three
// products (y = x W, dx = dz W^T, dW = x^T dz) read x, W and dz from where they lie, W stored [in, out].
//
// One persistent CTA (or pair of CTAs) per SM (pair) walks the output tiles:
//   warp 0   (one lane) copies 64-deep operand blocks into a ring of shared-memory stages by TMA
//   warp 1   owns the tensor memory; one lane issues four tcgen05.mma a stage (of the pair's first CTA alone)
//   warps 2-9  take the finished accumulator out of tensor memory, 32 columns of a row per thread, apply the epilogue
//            and store; two accumulators, so that this runs under the next tile's products.
// A pair (cta_group::2) computes 256 rows x BN columns: each CTA holds its own 128 rows of A and half of B's, and the
// tensor cores of both read both halves, so an operand byte in shared memory serves twice as many products.
// Copies that serve a pair signal the first CTA's barrier; no multicast copies are used.
//
// Every wait is bounded (2 s): whoever gives up sets the call's status word and its CTA's flag, all roles stop, copies
// and products under way are waited for (again with a limit), tensor memory is freed and the kernel returns.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "checkpoint8.cuh"
#include "tc_gemm.cuh"

namespace dynbatch {
namespace lg {

constexpr int kRows = 128;             // rows of A a CTA holds = its tensor-memory lanes
constexpr int kBlockK = 64;            // bf16 in a 128-byte swizzled row
constexpr int kEpilogueWarps = 8;      // two per tensor-memory lane quarter, half of the tile's columns each
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kMaxProblems = 3;
constexpr int kChunk = 32;             // columns of a row that a thread takes at once

enum Epilogue {
    kEpiStore = 0,      // out = act(acc + bias) + addend, acc + bias kept if wanted
    kEpiGated = 1,      // two accumulators side by side: out = act(gate) * up, both kept if wanted
    kEpiGatedGrad = 2   // acc = dh: with gate and up as kept, d_gate, d_up and h
};

struct Kept {                    // a tensor [M, N] as it is held for the backward pass
    void* data = nullptr;        // bf16 or e4m3 codes, N per row; nullptr: not kept
    uint8_t* scale = nullptr;    // e4m3: ceil(N / 32) bytes per row
};

struct EpilogueArgs {
    void* out = nullptr;         // kEpiStore: [M, N]; kEpiGated: h; kEpiGatedGrad: h
    long long out_pitch = 0;
    const __nv_bfloat16* bias = nullptr;
    const __nv_bfloat16* addend = nullptr;
    long long addend_pitch = 0;
    Kept kept[2];                // kEpiStore: [0]; the others: gate, up
    __nv_bfloat16* d_gate = nullptr;   // kEpiGatedGrad
    __nv_bfloat16* d_up = nullptr;
    long long d_pitch = 0;
    int kept_e4m3 = 0;
    int out_f32 = 0;
    int act = DB_ACT_NONE;
};

struct Problem {
    CUtensorMap a[2], b[2];      // the reduction's two sources; kEpiGated: b[0] gate's and b[1] up's weights
    int M, N;                    // output rows and columns
    int blocks0, blocks;         // 64-deep blocks of the first source, and of both
    int m_tiles, n_tiles;
    long long partial;           // first float of this problem's partial sums
    EpilogueArgs e;
};

struct GemmArgs {
    Problem p[kMaxProblems];
    int tile_start[kMaxProblems + 1];   // first tile of a problem, and their number; a tile for each split
    int problems;
    int splits, blocks_per_split;       // splits > 1: tiles leave as fp32 partial sums, folded by combine_kernel
    float* partials;                    // [problem][split][gate, up][M][columns rounded up to 32]
    int* status;
    int clear_status;                   // the first CTA zeroes *status
};

// ------------------------------------------------------------------------------------------------ 32 values of a row
__device__ __forceinline__ bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

__device__ __forceinline__ void unpack2(uint32_t two, float& a, float& b) {
    a = __uint_as_float(two << 16);
    b = __uint_as_float(two & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
// n of the 32 values exist; the others come back as zero
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, int n, float (&v)[kChunk]) {
    if (n == kChunk && aligned_to(p, 16)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = *(reinterpret_cast<const uint4*>(p) + i);
            unpack2(q.x, v[8 * i + 0], v[8 * i + 1]);
            unpack2(q.y, v[8 * i + 2], v[8 * i + 3]);
            unpack2(q.z, v[8 * i + 4], v[8 * i + 5]);
            unpack2(q.w, v[8 * i + 6], v[8 * i + 7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
    }
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, int n, const float (&v)[kChunk]) {
    if (n == kChunk && aligned_to(p, 16)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(reinterpret_cast<uint4*>(p) + i) = make_uint4(pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
                                                            pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7]));
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = __float2bfloat16_rn(v[i]);
    }
}
__device__ __forceinline__ void store_row(float* p, int n, const float (&v)[kChunk]) {
    if (n == kChunk && aligned_to(p, 16)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) *(reinterpret_cast<float4*>(p) + i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void keep_row(const Kept& k, int e4m3, long long row, int col, int N, int n, const float (&x)[kChunk]) {
    if (!e4m3) {
        store_row(static_cast<__nv_bfloat16*>(k.data) + row * N + col, n, x);
        return;
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
        if (i < n) top = fmaxf(top, ck8::finite_magnitude(x[i]));
    const uint32_t byte = ck8::scale_byte(top);
    const float inverse = ck8::scale_inverse(byte);
    k.scale[row * ((N + kChunk - 1) / kChunk) + col / kChunk] = static_cast<uint8_t>(byte);
    uint32_t c[8];
    if (byte < ck8::kTopByte) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = ck8::codes4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], inverse);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            c[i] = ck8::codes4(ck8::hold_finite(x[4 * i]), ck8::hold_finite(x[4 * i + 1]), ck8::hold_finite(x[4 * i + 2]),
                               ck8::hold_finite(x[4 * i + 3]), inverse);
    }
    uint8_t* p = static_cast<uint8_t*>(k.data) + row * N + col;
    if (n == kChunk && aligned_to(p, 16)) {
        *reinterpret_cast<uint4*>(p) = make_uint4(c[0], c[1], c[2], c[3]);
        *(reinterpret_cast<uint4*>(p) + 1) = make_uint4(c[4], c[5], c[6], c[7]);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = static_cast<uint8_t>(c[i / 4] >> (8 * (i % 4)));
    }
}
__device__ __forceinline__ void kept_row(const Kept& k, int e4m3, long long row, int col, int N, int n, float (&v)[kChunk]) {
    if (!e4m3) {
        load_row(static_cast<const __nv_bfloat16*>(k.data) + row * N + col, n, v);
        return;
    }
    const uint8_t* p = static_cast<const uint8_t*>(k.data) + row * N + col;
    const float scale = ck8::scale_value(k.scale[row * ((N + kChunk - 1) / kChunk) + col / kChunk]);
    uint32_t c[8];
    if (n == kChunk && aligned_to(p, 16)) {
        const uint4 q0 = *reinterpret_cast<const uint4*>(p), q1 = *(reinterpret_cast<const uint4*>(p) + 1);
        c[0] = q0.x; c[1] = q0.y; c[2] = q0.z; c[3] = q0.w;
        c[4] = q1.x; c[5] = q1.y; c[6] = q1.z; c[7] = q1.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * i + j < n) c[i] |= static_cast<uint32_t>(p[4 * i + j]) << (8 * j);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 a = ck8::values2(c[i]), b = ck8::values2(c[i] >> 16);
        v[4 * i + 0] = a.x * scale; v[4 * i + 1] = a.y * scale;
        v[4 * i + 2] = b.x * scale; v[4 * i + 3] = b.y * scale;
    }
}

// ------------------------------------------------------------------------------------------------ activations
// silu(z) = z s, s = 1 / (1 + e^-z);  gelu(z) = z P(z), P the normal distribution function.  The fast exponential and
// quotient are off by a few 2^-23 of a value that is rounded to 2^-9.
__device__ __forceinline__ float act_value(float z, int act) {
    if (act == DB_ACT_SILU) return z * __fdividef(1.f, 1.f + __expf(-z));
    if (act == DB_ACT_GELU) return z * (0.5f + 0.5f * erff(z * 0.70710678f));
    if (act == DB_ACT_RELU) return z < 0.f ? 0.f : z;
    return z;
}
__device__ __forceinline__ void act_value_slope(float z, int act, float& value, float& slope) {
    if (act == DB_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        value = z * s;
        slope = s * (1.f + z * (1.f - s));
    } else if (act == DB_ACT_GELU) {
        const float p = 0.5f + 0.5f * erff(z * 0.70710678f);
        value = z * p;
        slope = p + z * 0.39894228f * __expf(-0.5f * z * z);
    } else if (act == DB_ACT_RELU) {
        value = z < 0.f ? 0.f : z;
        slope = z <= 0.f ? 0.f : 1.f;
    } else {
        value = z;
        slope = 1.f;
    }
}
// The branch on the activation is taken once for a row, not for each value.
__device__ __forceinline__ void act_row(float (&v)[kChunk], int act) {
    if (act == DB_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = act_value(v[i], DB_ACT_SILU);
    } else if (act == DB_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = act_value(v[i], DB_ACT_GELU);
    } else if (act == DB_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = act_value(v[i], DB_ACT_RELU);
    }
}
template <int ACT>
__device__ __forceinline__ void gated_grad_row(const float (&dh)[kChunk], float (&gate)[kChunk], float (&up)[kChunk], float (&h)[kChunk]) {
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        float a, slope;
        act_value_slope(gate[i], ACT, a, slope);
        h[i] = a * up[i];
        gate[i] = dh[i] * up[i] * slope;
        up[i] = dh[i] * a;
    }
}

// n >= 1 columns of row `row` from column `col` (a multiple of 32): v the accumulator (kEpiGated: gate's), u up's.
template <int EPI>
__device__ __forceinline__ void epilogue_row(const EpilogueArgs& e, long long row, int col, int N, int n, float (&v)[kChunk],
                                             float (&u)[kChunk]) {
    if (EPI == kEpiStore) {
        if (e.bias) {
            float b[kChunk];
            load_row(e.bias + col, n, b);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] += b[i];
        }
        if (e.kept[0].data) keep_row(e.kept[0], e.kept_e4m3, row, col, N, n, v);
        act_row(v, e.act);
        if (e.addend) {
            float r[kChunk];
            load_row(e.addend + row * e.addend_pitch + col, n, r);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] += r[i];
        }
        if (e.out_f32) store_row(static_cast<float*>(e.out) + row * e.out_pitch + col, n, v);
        else store_row(static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col, n, v);
    } else if (EPI == kEpiGated) {
        if (e.kept[0].data) {
            keep_row(e.kept[0], e.kept_e4m3, row, col, N, n, v);
            keep_row(e.kept[1], e.kept_e4m3, row, col, N, n, u);
        }
        act_row(v, e.act);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] *= u[i];
        store_row(static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col, n, v);
    } else {
        float gate[kChunk];
        kept_row(e.kept[0], e.kept_e4m3, row, col, N, n, gate);
        kept_row(e.kept[1], e.kept_e4m3, row, col, N, n, u);
        float h[kChunk];
        if (e.act == DB_ACT_SILU) gated_grad_row<DB_ACT_SILU>(v, gate, u, h);
        else if (e.act == DB_ACT_GELU) gated_grad_row<DB_ACT_GELU>(v, gate, u, h);
        else if (e.act == DB_ACT_RELU) gated_grad_row<DB_ACT_RELU>(v, gate, u, h);
        else gated_grad_row<DB_ACT_NONE>(v, gate, u, h);
        store_row(e.d_gate + row * e.d_pitch + col, n, gate);
        store_row(e.d_up + row * e.d_pitch + col, n, u);
        store_row(static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col, n, h);
    }
}

// ------------------------------------------------------------------------------------------------ PTX wrappers
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t columns) {
    if (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tc::tmem_alloc(slot, columns);
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t columns) {
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else tc::tmem_dealloc(base, columns);
}
template <int CG>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier, in both CTAs of a pair, once all products issued so far by this thread have finished.
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(tc::smem_u32(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
    else
        tc::mma_commit(bar);
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of the same shared-memory word in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first_cta(const void* p) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(0));
    return a;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(tc::smem_u32(bar)), "r"(bytes) : "memory");
}
// One box; x counts bf16 of the contiguous dimension and is a multiple of 64 here (128 bytes).
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Operand tile with the reduction contiguous: rows of 64 bf16, 128-byte swizzle, 8-row groups 1024 bytes apart.
// Output index contiguous: blocks of 64 output indices x 64 reduction rows of 128 bytes; the next 64 output indices start
// 8192 bytes on (leading offset), the next 8 reduction rows 1024 (stride offset).
template <bool MN>
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    uint64_t d = tc::smem_desc_k_sw128(addr);
    if (MN) d += static_cast<uint64_t>((8192 >> 4) - 1) << 16;
    return d;
}
__host__ __device__ constexpr uint32_t instr_desc_bf16(int M, int N, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) |
           (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// ------------------------------------------------------------------------------------------------ tiles
template <int CG, int BN>
struct Shape {
    static constexpr int kTileM = kRows * CG;
    static constexpr int kBRows = BN / CG;                   // rows of B in one CTA
    static constexpr int kABytes = kRows * 128;
    static constexpr int kBBytes = kBRows * 128;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = 196608 / kStageBytes;     // 192 KB: six stages of 32 KB, eight of 24 KB
    static constexpr int kSmemBytes = kStages * kStageBytes + 1024;
    static constexpr uint32_t kTmemColumns = 2 * BN;         // two accumulators
    static_assert(kTmemColumns <= 512 && (kTmemColumns & (kTmemColumns - 1)) == 0 && kTmemColumns >= 32, "a power of two up to 512");
    static_assert(kBRows >= 64 && BN % 64 == 0, "whole blocks of 64 output indices");
};

struct Tile { int problem, split, m, n; };

// Tiles in an order that keeps those under way at one time in a compact part of the output: bands of 8 row tiles,
// column by column (the operands they share then come from L2).
__device__ __forceinline__ Tile decode(const GemmArgs& g, int t) {
    Tile r;
    r.problem = 0;
    while (r.problem + 1 < g.problems && t >= g.tile_start[r.problem + 1]) ++r.problem;
    const Problem& p = g.p[r.problem];
    t -= g.tile_start[r.problem];
    const int per_split = p.m_tiles * p.n_tiles;
    r.split = t / per_split;
    t -= r.split * per_split;
    constexpr int kBand = 8;
    const int band = t / (kBand * p.n_tiles), first = band * kBand;
    const int rows = min(kBand, p.m_tiles - first);
    t -= band * kBand * p.n_tiles;
    r.n = t / rows;
    r.m = first + (t - r.n * rows);
    return r;
}
// Blocks of the tile's reduction: [begin, end)
__device__ __forceinline__ void k_range(const GemmArgs& g, const Tile& t, int& begin, int& end) {
    begin = t.split * g.blocks_per_split;
    end = min(g.p[t.problem].blocks, begin + g.blocks_per_split);
}
__host__ __device__ constexpr long long partial_pitch(long long N) { return (N + kChunk - 1) / kChunk * kChunk; }

template <int CG, int BN, bool A_MN, bool B_MN, int EPI>
__global__ void __launch_bounds__(kThreads, 1)
layer_gemm_kernel(const __grid_constant__ GemmArgs g) {
    using S = Shape<CG, BN>;
    constexpr int kTileN = EPI == kEpiGated ? BN / 2 : BN;   // output columns of a tile
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[S::kStages];    // a stage's copies have landed (first CTA's is used)
    __shared__ __align__(8) uint64_t empty_bar[S::kStages];   // the products reading it have finished
    __shared__ __align__(8) uint64_t ready_bar[2];            // an accumulator is complete
    __shared__ __align__(8) uint64_t taken_bar[2];            // ... and has been read out (first CTA's is used)
    __shared__ __align__(8) uint64_t drain_bar;               // after a time-out: all products issued have finished
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;

    unsigned char* tiles = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
    const int total = g.tile_start[g.problems];

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < S::kStages; ++s) {
            tc::mbar_init(&full_bar[s], 1);
            tc::mbar_init(&empty_bar[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&ready_bar[i], 1);
            tc::mbar_init(&taken_bar[i], CG * kEpilogueWarps);
        }
        tc::mbar_init(&drain_bar, 1);
        tc::fence_barrier_init();
    }
    if (warp == 1) tmem_alloc<CG>(&tmem_slot, S::kTmemColumns);
    tc::tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tmem_slot;

    // Nothing above touches global memory.  The successor is released only when the predecessor has finished, so at
    // most one kernel waits in the wings and everything before this one is complete.
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    if (g.clear_status && blockIdx.x == 0 && tid == 0) *g.status = 0;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;                                       // stages filled so far
            bool ok = true;
            for (int t = worker; t < total && ok; t += workers) {
                const Tile tile = decode(g, t);
                const Problem& p = g.p[tile.problem];
                int k, k_end;
                k_range(g, tile, k, k_end);
                const int m0 = tile.m * S::kTileM + static_cast<int>(rank) * kRows;
                // what this CTA holds of B: gated, a pair's CTAs take one weight each, a single CTA half of both
                const int n0 = tile.n * kTileN + (EPI == kEpiGated ? 0 : static_cast<int>(rank) * S::kBRows);
                for (; k < k_end; ++k, ++it) {
                    const int s = it % S::kStages;
                    if (!(ok = tc::mbar_wait(&empty_bar[s], ((it / S::kStages) & 1) ^ 1, &abort_flag, g.status, 0x301))) break;
                    const uint32_t bar = CG == 2 ? in_first_cta(&full_bar[s]) : tc::smem_u32(&full_bar[s]);
                    if (rank == 0) expect_tx(&full_bar[s], CG * S::kStageBytes);
                    const int source = k >= p.blocks0;
                    const int k0 = (source ? k - p.blocks0 : k) * kBlockK;
                    const uint32_t a = tc::smem_u32(tiles + s * S::kStageBytes), b = a + S::kABytes;
                    if (A_MN) {
#pragma unroll
                        for (int c = 0; c < kRows / 64; ++c) tma_load<CG>(a + c * 8192, &p.a[source], m0 + 64 * c, k0, bar);
                    } else {
                        tma_load<CG>(a, &p.a[source], k0, m0, bar);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int c = 0; c < S::kBRows / 64; ++c) {
                            constexpr int kHalf = S::kBRows / 128;   // blocks of 64 a single CTA takes of each weight
                            const CUtensorMap* map = EPI != kEpiGated ? &p.b[source] : CG == 2 ? &p.b[rank] : &p.b[c >= kHalf];
                            const int x = EPI == kEpiGated && CG == 1 ? n0 + 64 * (c % (kHalf ? kHalf : 1)) : n0 + 64 * c;
                            tma_load<CG>(b + c * 8192, map, x, k0, bar);
                        }
                    } else {
                        tma_load<CG>(b, &p.b[source], k0, n0, bar);
                    }
                }
            }
            if (ok) {
                // every product that reads this CTA's stages has finished, and its arrival has reached this CTA
                for (int i = it > S::kStages ? it - S::kStages : 0; i < it && ok; ++i)
                    ok = tc::mbar_wait(&empty_bar[i % S::kStages], (i / S::kStages) & 1, &abort_flag, g.status, 0x302);
            }
            if (!ok) {
                // copies under way land within microseconds; their barrier may be the other CTA's
                const unsigned long long t0 = tc::global_ns();
                while (tc::global_ns() - t0 < 5000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = instr_desc_bf16(S::kTileM, BN, A_MN, B_MN);
            constexpr uint32_t kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;   // 16 of the reduction
            int it = 0, n = 0;
            bool ok = true;
            for (int t = worker; t < total && ok; t += workers, ++n) {
                const Tile tile = decode(g, t);
                int k, k_end;
                k_range(g, tile, k, k_end);
                const int buf = n & 1;
                if (!(ok = tc::mbar_wait(&taken_bar[buf], ((n >> 1) & 1) ^ 1, &abort_flag, g.status, 0x303))) break;
                tc::tc_fence_after();
                const uint32_t acc = tmem + buf * BN;
                for (bool first = true; k < k_end; ++k, ++it, first = false) {
                    const int s = it % S::kStages;
                    if (!(ok = tc::mbar_wait(&full_bar[s], (it / S::kStages) & 1, &abort_flag, g.status, 0x304))) break;
                    tc::tc_fence_after();
                    const uint32_t a = tc::smem_u32(tiles + s * S::kStageBytes);
                    const uint64_t da = smem_desc<A_MN>(a), db = smem_desc<B_MN>(a + S::kABytes);
#pragma unroll
                    for (int i = 0; i < kBlockK / 16; ++i)
                        mma_bf16<CG>(acc, da + i * kStepA, db + i * kStepB, idesc, !(first && i == 0));
                    mma_commit<CG>(&empty_bar[s]);
                }
                if (ok) mma_commit<CG>(&ready_bar[buf]);
            }
            if (!ok) {
                mma_commit<CG>(&drain_bar);
                unsigned long long t0 = tc::global_ns();
                while (!tc::mbar_try_wait(&drain_bar, 0) && tc::global_ns() - t0 < tc::kWaitLimitNs) {}
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        int n = 0;
        for (int t = worker; t < total; t += workers, ++n) {
            const Tile tile = decode(g, t);
            const Problem& p = g.p[tile.problem];
            const int buf = n & 1;
            if (!__all_sync(0xFFFFFFFFu, tc::mbar_wait(&ready_bar[buf], (n >> 1) & 1, &abort_flag, g.status, 0x305))) break;
            tc::tc_fence_after();
            const long long row = static_cast<long long>(tile.m) * S::kTileM + rank * kRows + quarter * 32 + lane;
            const uint32_t acc = tmem + buf * BN + (static_cast<uint32_t>(quarter * 32) << 16);
            constexpr int kPerWarp = kTileN / 2;
            const int N = p.N;
#pragma unroll 1
            for (int c = 0; c < kPerWarp; c += kChunk) {
                __syncwarp();                                  // rows past the end rejoin for the next read
                const int in_tile = half * kPerWarp + c, col = tile.n * kTileN + in_tile;
                if (col >= N) break;                           // the same for the whole warp
                uint32_t raw[kChunk];
                float v[kChunk], u[kChunk];
                tc::tmem_load32(acc + in_tile, raw);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[i] = __uint_as_float(raw[i]);
                if (EPI == kEpiGated) {
                    tc::tmem_load32(acc + kTileN + in_tile, raw);
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) u[i] = __uint_as_float(raw[i]);
                }
                if (row >= p.M) continue;
                if (g.splits > 1) {
                    const long long pitch = partial_pitch(N), plane = p.M * pitch;
                    float* to = g.partials + p.partial + tile.split * plane * (EPI == kEpiGated ? 2 : 1) + row * pitch + col;
                    store_row(to, kChunk, v);
                    if (EPI == kEpiGated) store_row(to + plane, kChunk, u);
                } else {
                    epilogue_row<EPI>(p.e, row, col, N, min(kChunk, N - col), v, u);
                }
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) arrive_cluster(in_first_cta(&taken_bar[buf]));
                else tc::mbar_arrive(&taken_bar[buf]);
            }
        }
        __syncwarp();
    }
    tc::tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after();
        tmem_dealloc<CG>(tmem, S::kTmemColumns);
    }
}

// Folds the partial sums of a split reduction in split order and applies the epilogue; a thread has 32 columns of a row.
template <int EPI>
__global__ void __launch_bounds__(128)
combine_kernel(const __grid_constant__ GemmArgs g) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const Problem& p = g.p[blockIdx.y];
    const long long pitch = partial_pitch(p.N), plane = p.M * pitch, chunks = pitch / kChunk;
    const long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (i >= p.M * chunks) return;
    const long long row = i / chunks;
    const int col = static_cast<int>(i - row * chunks) * kChunk;
    const long long step = plane * (EPI == kEpiGated ? 2 : 1);
    const float* from = g.partials + p.partial + row * pitch + col;
    float v[kChunk], u[kChunk];
#pragma unroll
    for (int j = 0; j < kChunk; ++j) v[j] = u[j] = 0.f;
    for (int s = 0; s < g.splits; ++s) {
#pragma unroll
        for (int j = 0; j < kChunk; j += 4) {
            const float4 q = *reinterpret_cast<const float4*>(from + s * step + j);
            v[j] += q.x; v[j + 1] += q.y; v[j + 2] += q.z; v[j + 3] += q.w;
            if (EPI == kEpiGated) {
                const float4 r = *reinterpret_cast<const float4*>(from + s * step + plane + j);
                u[j] += r.x; u[j + 1] += r.y; u[j + 2] += r.z; u[j + 3] += r.w;
            }
        }
    }
    epilogue_row<EPI>(p.e, row, col, p.N, static_cast<int>(min(static_cast<long long>(kChunk), static_cast<long long>(p.N) - col)), v, u);
}

}  // namespace lg
}  // namespace dynbatch
