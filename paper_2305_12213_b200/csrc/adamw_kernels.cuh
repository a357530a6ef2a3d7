// Device code of the AdamW step over a tensor list and of the global norm of the weighted gradient
// (Section 3.1, Eq. 2 for the aggregate; AdamW and the clipping are what language models train with).
//
// Work is laid out in blocks of 256 consecutive elements of one tensor, one warp each: the unit that shares a
// scale when the moments are held in 8 bits.  A CTA's eight warps take one tile of eight blocks; a record in
// device memory holds the tile's pointers.  Lanes own eight elements: consecutive ones when every buffer of the
// tensor is aligned (one 32-byte access for fp32, 16 for bf16, 8 for e4m3), otherwise every 32nd one, element by
// element.  What is computed for an element does not depend on which lane has it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <cstdint>

#include "agg_device.cuh"
#include "dynbatch.h"

namespace dynbatch {
namespace adamw {

constexpr int kThreads = 256;
constexpr int kLaneElems = 8;
constexpr int kWarpElems = DB_ADAMW_BLOCK;                       // 32 lanes x 8 elements
constexpr int kTile = kThreads * kLaneElems;
static_assert(kWarpElems == 32 * kLaneElems, "one warp per block of elements");

// Words of 8 bytes of a tile's record; the K gradient pointers follow at kRecGrads.
enum RecordWord {
    kRecParam = 0, kRecFirst, kRecSecond, kRecCount,             // count | flags << 32
    kRecFirstScale, kRecSecondScale, kRecCopy, kRecDecay,        // bits of the fp32 weight decay
    kRecPosition, kRecSpare, kRecGrads
};
enum NormRecordWord { kNormCount = 0, kNormSpare, kNormGrads };
constexpr int kStateAligned = 1, kGradsAligned = 2;

struct Source {                  // where the weighted gradient comes from
    const long long* recs;       // records, `stride` words apart
    float lambda[DB_MAX_K];      // weights of the active workers (b_k > 0), in worker order
    unsigned char worker[DB_MAX_K];   // their indexes
    int K;                       // how many
    int stride;
    long long tiles;
    float* staged;               // kTile fp32 aggregates for each tile, or NULL
};

struct NormArgs {
    Source src;
    int count_word, grads_word;
    double* partials;            // one per CTA
};

struct StepArgs {
    Source src;
    double* partials;            // norm partials (NORM only)
    const float* factor;         // clipping factor in device memory (CLIP only)
    float beta1, one_minus_beta1, beta2, one_minus_beta2;
    float step_size;             // lr / (1 - beta1^t)
    float inv_sqrt_c2;           // 1 / sqrt(1 - beta2^t)
    float eps, lr;
    uint32_t key0, key1;
};

// ---- memory access of one lane's eight elements --------------------------------------------------
// ALIGNED: elements 8 lane .. 8 lane + 7.  Otherwise elements lane + 32 i, those below n.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    asm volatile("ld.global.cs.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    asm volatile("st.global.cs.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]),
                 "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
}

template <bool ALIGNED>
__device__ __forceinline__ void load_f32(const float* p, int lane, int n, float (&x)[8]) {
    if (ALIGNED) {
        load8(p + 8 * lane, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = lane + 32 * i < n ? __ldcs(p + lane + 32 * i) : 0.0f;
    }
}
template <bool ALIGNED>
__device__ __forceinline__ void store_f32(float* p, int lane, int n, const float (&x)[8]) {
    if (ALIGNED) {
        store8(p + 8 * lane, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < n) __stcs(p + lane + 32 * i, x[i]);
    }
}

// Raw gradient vectors, widened only when they are used, so that several workers' loads are in flight at once.
template <typename GT> struct GradRaw;
template <> struct GradRaw<float> {
    float x[8];
    template <bool ALIGNED>
    __device__ __forceinline__ void load(const void* base, int lane, int n) {
        load_f32<ALIGNED>(static_cast<const float*>(base), lane, n, x);
    }
    __device__ __forceinline__ float get(int i) const { return x[i]; }
};
template <> struct GradRaw<__nv_bfloat16> {
    uint32_t x[4];               // bf16 is the high half of a binary32: widening is a shift, exact
    template <bool ALIGNED>
    __device__ __forceinline__ void load(const void* base, int lane, int n) {
        const uint16_t* p = static_cast<const uint16_t*>(base);
        if (ALIGNED) {
            const uint4 r = __ldcs(reinterpret_cast<const uint4*>(p + 8 * lane));
            x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = lane + 64 * i;
                const uint32_t lo = j < n ? __ldcs(p + j) : 0u, hi = j + 32 < n ? __ldcs(p + j + 32) : 0u;
                x[i] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
    }
};

// g = sum over the active workers of lambda_k g_k: fp32 FMAs, k ascending, from zero.  KU workers' loads at once.
template <typename GT, int KU, bool ALIGNED>
__device__ __forceinline__ void aggregate(const Source& s, const long long* grads, int offset, int lane, int n,
                                          float (&g)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 0.0f;
    for (int k0 = 0; k0 < s.K; k0 += KU) {
        GradRaw<GT> raw[KU];
#pragma unroll
        for (int j = 0; j < KU; ++j)
            if (k0 + j < s.K)
                raw[j].template load<ALIGNED>(reinterpret_cast<const GT*>(__ldg(grads + s.worker[k0 + j])) + offset, lane, n);
#pragma unroll
        for (int j = 0; j < KU; ++j) {
            if (k0 + j < s.K) {
                const float w = s.lambda[k0 + j];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = fmaf(w, raw[j].get(i), g[i]);
            }
        }
    }
}

// Sum of the squares of a lane's eight aggregates.  In fp32 where every square that matters is a normal number,
// in fp64 otherwise (a finite gradient beyond 1.8e19 has no fp32 square).
__device__ __forceinline__ double sum_squares(const float (&g)[8]) {
    float top = 0.0f, part = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top = fmaxf(top, fabsf(g[i]));
        part = fmaf(g[i], g[i], part);
    }
    if (top < 1e15f && (top > 1e-15f || top == 0.0f)) return static_cast<double>(part);
    double wide = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) wide = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), wide);
    return wide;
}

// ---- 8-bit moments --------------------------------------------------------------------------------
// 32 random bits for an element: two rounds of a 32 x 32 -> 64-bit multiply whose halves are folded together,
// keyed by the call's seed and step.
__device__ __forceinline__ uint32_t fold_multiply(uint32_t x, uint32_t m) {
    const uint64_t z = static_cast<uint64_t>(x) * m;
    return static_cast<uint32_t>(z >> 32) ^ static_cast<uint32_t>(z);
}
__device__ __forceinline__ uint32_t random_bits(uint32_t position_low, uint32_t key0, uint32_t key1) {
    return fold_multiply(fold_multiply(position_low ^ key0, 0xAC4C1B51u) ^ key1, 0xD6E8FEB5u);
}

// e4m3 code of magnitude y in [0, 448], taken up to the next value with probability (distance below y) / (step):
// `chance` has 16 random bits.  Scaled by 2^-120, the 8-bit type's exponents (subnormals included) are binary32's
// lowest ones, so one step is 2^20 units of the bit pattern: add the chance below it and cut off.
__device__ __forceinline__ uint32_t encode(float y, uint32_t chance) {
    const uint32_t bits = __float_as_uint(y * 0x1p-120f) + (chance << 4);
    return min(bits >> 20, 0x7eu);
}

// Block scale: a = max |x| over the warp's 256 elements.  Returns 448 / s for s = max(a, 2^-100) and s / 448; a
// block with a value that is not finite gets a NaN scale and keep = 0 (codes are masked to zero).
struct BlockScale {
    float to_code, scale;
    uint32_t keep;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t lane_top) {
    const uint32_t top = max(__reduce_max_sync(0xffffffffu, lane_top), 0x0d800000u);      // bits of 2^-100
    const bool finite = top < 0x7f800000u;
    const float s = __uint_as_float(top);
    BlockScale r;
    r.to_code = 448.0f / s;
    r.scale = finite ? s / 448.0f : __uint_as_float(0x7fffffffu);
    r.keep = finite ? 0xffffffffu : 0u;
    return r;
}

template <bool ALIGNED>
__device__ __forceinline__ void load_codes(const uint8_t* p, int lane, int n, float scale, float (&x)[8]) {
    uint32_t c[2] = {0u, 0u};
    if (ALIGNED) {
        const uint2 r = __ldcs(reinterpret_cast<const uint2*>(p + 8 * lane));
        c[0] = r.x; c[1] = r.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < n) c[i >> 2] |= static_cast<uint32_t>(__ldcs(p + lane + 32 * i)) << (8 * (i & 3));
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(c[i >> 2] >> (8 * (i & 3))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x[i] = f.x * scale;
        x[i + 1] = f.y * scale;
    }
}
template <bool ALIGNED>
__device__ __forceinline__ void store_codes(uint8_t* p, int lane, int n, const uint32_t (&c)[2]) {
    if (ALIGNED) {
        __stcs(reinterpret_cast<uint2*>(p + 8 * lane), make_uint2(c[0], c[1]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < n) p[lane + 32 * i] = static_cast<uint8_t>(c[i >> 2] >> (8 * (i & 3)));
    }
}

// ---- one block of elements ------------------------------------------------------------------------
template <typename GT, int KU, bool STATE8, bool CLIP, bool NORM, bool ALIGNED>
__device__ __forceinline__ void step_block(const StepArgs& a, const long long* rec, long long tile, int offset, int lane,
                                           int n, float factor, double& sq) {
    float* param = reinterpret_cast<float*>(__ldg(rec + kRecParam)) + offset;
    float p[8], m[8], u[8], g[8];
    load_f32<ALIGNED>(param, lane, n, p);
    const long long first = __ldg(rec + kRecFirst), second = __ldg(rec + kRecSecond);
    float *first_scale = nullptr, *second_scale = nullptr;
    if (STATE8) {
        first_scale = reinterpret_cast<float*>(__ldg(rec + kRecFirstScale)) + offset / kWarpElems;
        second_scale = reinterpret_cast<float*>(__ldg(rec + kRecSecondScale)) + offset / kWarpElems;
        load_codes<ALIGNED>(reinterpret_cast<const uint8_t*>(first) + offset, lane, n, *first_scale, m);
        load_codes<ALIGNED>(reinterpret_cast<const uint8_t*>(second) + offset, lane, n, *second_scale, u);
    } else {
        load_f32<ALIGNED>(reinterpret_cast<const float*>(first) + offset, lane, n, m);
        load_f32<ALIGNED>(reinterpret_cast<const float*>(second) + offset, lane, n, u);
    }
    if (CLIP && a.src.staged)
        load_f32<ALIGNED>(a.src.staged + tile * kTile + offset, lane, n, g);
    else
        aggregate<GT, KU, ALIGNED>(a.src, rec + kRecGrads, offset, lane, n, g);
    if (NORM) sq += sum_squares(g);

    const float decay = 1.0f - a.lr * __uint_as_float(static_cast<uint32_t>(__ldg(rec + kRecDecay)));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float h = CLIP ? g[i] * factor : g[i];
        m[i] = fmaf(a.beta1, m[i], a.one_minus_beta1 * h);
        u[i] = fmaf(a.beta2, u[i], a.one_minus_beta2 * (h * h));
        p[i] = fmaf(-a.step_size, m[i] / fmaf(sqrtf(u[i]), a.inv_sqrt_c2, a.eps), p[i] * decay);
    }
    store_f32<ALIGNED>(param, lane, n, p);
    if (const long long copy = __ldg(rec + kRecCopy)) {
        __nv_bfloat16* w = reinterpret_cast<__nv_bfloat16*>(copy) + offset;
        if (ALIGNED) {
            uint4 r;
            __nv_bfloat162 h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(p[2 * i], p[2 * i + 1]);
            r.x = *reinterpret_cast<uint32_t*>(&h[0]); r.y = *reinterpret_cast<uint32_t*>(&h[1]);
            r.z = *reinterpret_cast<uint32_t*>(&h[2]); r.w = *reinterpret_cast<uint32_t*>(&h[3]);
            *reinterpret_cast<uint4*>(w + 8 * lane) = r;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (lane + 32 * i < n) w[lane + 32 * i] = __float2bfloat16_rn(p[i]);
        }
    }
    if (STATE8) {
        uint32_t top_m = 0u, top_u = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!ALIGNED && lane + 32 * i >= n) continue;
            top_m = max(top_m, __float_as_uint(m[i]) & 0x7fffffffu);
            top_u = max(top_u, __float_as_uint(u[i]) & 0x7fffffffu);
        }
        const BlockScale sm = block_scale(top_m), su = block_scale(top_u);
        const long long position = __ldg(rec + kRecPosition) + offset;      // a multiple of 256: the high word is the block's
        const uint32_t low = static_cast<uint32_t>(position) + (ALIGNED ? 8 * lane : lane);
        const uint32_t key1 = a.key1 ^ (static_cast<uint32_t>(position >> 32) * 0x85EBCA6Bu);
        uint32_t cm[2] = {0u, 0u}, cu[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = random_bits(low + (ALIGNED ? i : 32 * i), a.key0, key1);
            const uint32_t em = encode(fabsf(m[i]) * sm.to_code, r & 0xffffu) | (__float_as_uint(m[i]) >> 24 & 0x80u);
            // a second moment that is not zero is never held as zero: the next step divides by its root
            const uint32_t eu = max(encode(u[i] * su.to_code, r >> 16), min(__float_as_uint(u[i]), 1u));
            cm[i >> 2] |= em << (8 * (i & 3));
            cu[i >> 2] |= eu << (8 * (i & 3));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            cm[i] &= sm.keep;
            cu[i] &= su.keep;
        }
        store_codes<ALIGNED>(reinterpret_cast<uint8_t*>(first) + offset, lane, n, cm);
        store_codes<ALIGNED>(reinterpret_cast<uint8_t*>(second) + offset, lane, n, cu);
        if (lane == 0) {
            *first_scale = sm.scale;
            *second_scale = su.scale;
        }
    } else {
        store_f32<ALIGNED>(reinterpret_cast<float*>(first) + offset, lane, n, m);
        store_f32<ALIGNED>(reinterpret_cast<float*>(second) + offset, lane, n, u);
    }
}

// One CTA per tile.
template <typename GT, int KU, bool STATE8, bool CLIP, bool NORM>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ StepArgs a) {
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const int lane = threadIdx.x & 31, offset = (threadIdx.x >> 5) * kWarpElems;
    const long long tile = blockIdx.x;
    const long long* rec = a.src.recs + tile * a.src.stride;
    const long long cf = __ldg(rec + kRecCount);
    const int n = static_cast<int>(cf & 0xffffffffLL) - offset, flags = static_cast<int>(cf >> 32);
    const float factor = CLIP ? __ldcg(a.factor) : 1.0f;
    double sq = 0.0;
    if (n > 0) {
        const bool aligned = flags & kStateAligned && (flags & kGradsAligned || (CLIP && a.src.staged));
        if (aligned && n >= kWarpElems)
            step_block<GT, KU, STATE8, CLIP, NORM, true>(a, rec, tile, offset, lane, kWarpElems, factor, sq);
        else
            step_block<GT, KU, STATE8, CLIP, NORM, false>(a, rec, tile, offset, lane, min(n, kWarpElems), factor, sq);
    }
    if (NORM) agg::store_norm_partial(a.partials, sq);
}

// The norm of the weighted gradient alone: a CTA takes tiles blockIdx.x, blockIdx.x + gridDim.x, ...; with a
// staging buffer it also leaves the aggregates there, for the step that follows.
template <typename GT, int KU>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ NormArgs a) {
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const int lane = threadIdx.x & 31, offset = (threadIdx.x >> 5) * kWarpElems;
    double sq = 0.0;
    for (long long tile = blockIdx.x; tile < a.src.tiles; tile += gridDim.x) {
        const long long* rec = a.src.recs + tile * a.src.stride;
        const long long cf = __ldg(rec + a.count_word);
        const int n = static_cast<int>(cf & 0xffffffffLL) - offset, flags = static_cast<int>(cf >> 32);
        if (n <= 0) continue;
        float g[8];
        float* staged = a.src.staged ? a.src.staged + tile * kTile + offset : nullptr;
        if (flags & kGradsAligned && n >= kWarpElems) {
            aggregate<GT, KU, true>(a.src, rec + a.grads_word, offset, lane, kWarpElems, g);
            if (staged) store8(staged + 8 * lane, g);
        } else {
            aggregate<GT, KU, false>(a.src, rec + a.grads_word, offset, lane, min(n, kWarpElems), g);
            if (staged) store_f32<false>(staged, lane, min(n, kWarpElems), g);
        }
        sq += sum_squares(g);
    }
    agg::store_norm_partial(a.partials, sq);
}

// Folds the partials: CTA c sums partials [c per, (c + 1) per).  The last stage (one CTA) writes the norm and the
// clipping factor max_norm / norm where the norm is larger than max_norm, else 1 (a NaN norm does not clip).
static __global__ void __launch_bounds__(1024) fold_kernel(const double* __restrict__ partials, long long n, int per,
                                                           double* __restrict__ sums, float* __restrict__ norm,
                                                           float* __restrict__ factor, float max_norm) {
    __shared__ double smem[32];
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const long long begin = static_cast<long long>(blockIdx.x) * per;
    const long long end = begin + per < n ? begin + per : n;
    double acc = 0.0;
    for (long long i = begin + threadIdx.x; i < end; i += blockDim.x) acc += __ldcg(partials + i);
    const double total = agg::block_sum(acc, smem);
    if (threadIdx.x != 0) return;
    if (sums) {
        sums[blockIdx.x] = total;
        return;
    }
    const double root = sqrt(total);
    if (norm) *norm = static_cast<float>(root);
    if (factor) *factor = root > static_cast<double>(max_norm) ? static_cast<float>(max_norm / root) : 1.0f;
}

}  // namespace adamw
}  // namespace dynbatch
