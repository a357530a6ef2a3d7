// Device code of the AdamW step over a tensor list and of the global norm of the weighted gradient
// (Section 3.1, Eq. 2 for the aggregate; AdamW and the clipping are what language models train with).
//
// Work is laid out in blocks of 256 consecutive elements of one tensor, one warp each: the unit that shares a
// scale when the moments are held in 8 bits.  A record in device memory holds the pointers of a run of up to
// `run` elements (a multiple of 2048, one step of a CTA's eight warps) of one tensor; a CTA takes a record.
// Lanes own eight consecutive elements (one 32-byte access for fp32, 16 for bf16, 8 for e4m3) where a tensor's states
// are aligned; its gradients, where they are not, reach their lanes through shared memory.
// A tensor whose states are off that grid goes element by element, and so does its last, shorter block (with 8-bit
// moments and aligned states that block comes through the ring like the others).  What is computed for an element does
// not depend on which lane has it.
//
// All three kernels are bound by the memory: a parameter costs K gradients + 24 bytes with 32-bit moments (19 instructions
// for one worker, 37 for eight), + 12 with 8-bit ones (55 and 97); the norm K gradients alone (101 for sixteen workers).
// Measured on B200, bytes counted once, against its copy rate of 6.56 TB/s:
//   32-bit, 470M parameters, one bf16 gradient, bf16 copy   1951 us   6.72 TB/s   1.03
//   32-bit, 25.6M, eight fp32 gradients                      213 us   6.72 TB/s   1.02
//    8-bit, 116M, one bf16 gradient, bf16 copy               289 us   6.44 TB/s   0.98
//    8-bit, 110M, eight bf16 gradients, bf16 copy             534 us   6.15 TB/s   0.94
//   norm, 110M, sixteen bf16 gradients                       589 us   5.93 TB/s   0.90
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <cstdint>
#include <type_traits>

#include "agg_device.cuh"
#include "dynbatch.h"

namespace dynbatch {
namespace adamw {

constexpr int kThreads = 256;
constexpr int kLaneElems = 8;
constexpr int kWarpElems = DB_ADAMW_BLOCK;                       // 32 lanes x 8 elements
constexpr int kSpan = kThreads * kLaneElems;                       // elements of a CTA's step
constexpr int kWarps = kThreads / 32;
constexpr int kNormThreads = kThreads / 2;                         // the norm kernel: two CTAs for a record
static_assert(kWarpElems == 32 * kLaneElems, "one warp per block of elements");

// Words of 8 bytes of a run's record; the K gradient pointers follow at kRecGrads.
enum RecordWord {
    kRecParam = 0, kRecFirst, kRecSecond, kRecCount,             // count | flags << 32
    kRecFirstScale, kRecSecondScale, kRecCopy, kRecDecay,        // bits of the fp32 weight decay
    kRecPosition, kRecGrads
};
enum NormRecordWord { kNormCount = 0, kNormPosition, kNormGrads };
constexpr int kStateAligned = 1, kGradsAligned = 2;              // flags: buffers aligned to a lane's vector

// Records ahead of a CTA's own that it asks the L2 for (a wave is some hundred): the data that streams through has
// evicted them, and a CTA that meets its record in DRAM starts 0.5 us later (norm of 110M, 16 workers: 692 -> 611 us).
constexpr long long kAhead = 512;
// Partials that a clipped step adds itself, every warp for itself, which takes the fold off the chain norm - fold - step
// (replayed, us, against the fold in the norm kernel's last CTA or behind it: 20,000 parameters 6.4 and 7.5; 246 partials
// 11.4 and 12.1; 490 from one fp32 gradient 18.7 and 16.7, from four 10.7 and 11.8 with 8-bit moments, 12.2 and 12.4 with
// 32-bit ones; 734 26.5 and 20.8); with more of them the reads cost more than the launch.
constexpr int kFoldInStep = 512;

struct Source {                  // where the weighted gradient comes from
    const long long* recs;       // records, `stride` words apart
    long long records;
    unsigned long long lambda[DB_MAX_K];   // weights of the active workers (b_k > 0), in worker order, as pairs
    unsigned char worker[DB_MAX_K];   // their indexes
    int K;                       // how many
    int stride;
    float* staged;               // fp32 aggregates by position (256 a block), or NULL
    unsigned long long one;      // a pair of ones, see add()
};

struct NormArgs {
    Source src;
    double* partials;            // one per CTA
    unsigned int* ticket;        // LAST: CTAs that have left their partial; 0 between launches
    float* norm;                 // or NULL
    float* factor;               // or NULL
    float max_norm;
};

struct StepArgs {
    Source src;
    double* partials;            // norm partials (NORM only)
    // CLIP: the clipping factor in device memory; or, where partial_count > 0, the norm's partials, which every warp
    // adds for itself (CTA 0 then writes the norm)
    const float* factor;
    int partial_count;
    float max_norm;
    float* norm;
    // pairs of fp32, both halves alike, as the packed arithmetic takes them
    unsigned long long beta1, one_minus_beta1, beta2, one_minus_beta2;
    unsigned long long minus_step_size;   // -lr / (1 - beta1^t)
    unsigned long long inv_sqrt_c2;       // 1 / sqrt(1 - beta2^t)
    unsigned long long eps;
    float lr;
    uint32_t key0, key1;
};

// ---- pairs of fp32 ---------------------------------------------------------------------------------
// Two elements in a 64-bit register: one instruction multiplies or adds both, each rounded on its own.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pack(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float lo(Pair x) { return __uint_as_float(static_cast<uint32_t>(x)); }
__device__ __forceinline__ float hi(Pair x) { return __uint_as_float(static_cast<uint32_t>(x >> 32)); }
__device__ __forceinline__ Pair both(float x) { return pack(x, x); }
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul_add(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// a + b, as an FMA with a one that the compiler does not know (`one`, both halves, comes from the host).  ptxas 12.9
// joins a packed product and a packed sum into one FMA, rounded once, even with .rn on both and --fmad=false
// (measured: 26 % of a b + c d then differ from the separately rounded sum); this it cannot join.
__device__ __forceinline__ Pair add(Pair a, Pair b, Pair one) { return mul_add(a, one, b); }

// Approximate square root and reciprocal (relative error 2^-23 each): they enter the parameter only, through a
// move that is a small part of it.  Both flush subnormals: a second moment below 2^-126 counts as 0 in the
// denominator; a denominator is 0 or normal, the host having raised a subnormal eps to the least normal number.
__device__ __forceinline__ float root(float x) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---- memory access of one lane's eight elements --------------------------------------------------
// ALIGNED: elements 8 lane .. 8 lane + 7.  Otherwise elements lane + 32 i, those below n.
template <bool ALIGNED>
__device__ __forceinline__ void load_f32(const float* p, int lane, int n, Pair (&x)[4]) {
    if (ALIGNED) {
        asm volatile("ld.global.cs.v4.b64 {%0,%1,%2,%3}, [%4];"
                     : "=l"(x[0]), "=l"(x[1]), "=l"(x[2]), "=l"(x[3])
                     : "l"(p + 8 * lane));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = lane + 64 * i;
            x[i] = pack(j < n ? __ldcs(p + j) : 0.0f, j + 32 < n ? __ldcs(p + j + 32) : 0.0f);
        }
    }
}
template <bool ALIGNED>
__device__ __forceinline__ void store_f32(float* p, int lane, int n, const Pair (&x)[4]) {
    if (ALIGNED) {
        asm volatile("st.global.cs.v4.b64 [%0], {%1,%2,%3,%4};" ::"l"(p + 8 * lane), "l"(x[0]), "l"(x[1]), "l"(x[2]), "l"(x[3])
                     : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = lane + 64 * i;
            if (j < n) __stcs(p + j, lo(x[i]));
            if (j + 32 < n) __stcs(p + j + 32, hi(x[i]));
        }
    }
}

// How a lane reads its eight gradients of a block: a vector of consecutive ones (kVector); a whole block off the
// vector grid, coalesced by words (kRows); element by element below n (kMasked).  kRows' and kMasked's fp32 lanes
// have elements lane + 32 i; kRows' bf16 lanes have the pairs 64 i + 2 lane.
enum Access { kVector, kRows, kMasked };

// Raw gradients, widened only when they are used, so that several workers' loads are in flight at once.
template <typename GT> struct GradRaw;
template <> struct GradRaw<float> {
    Pair x[4];
    template <Access A>
    __device__ __forceinline__ void load(const float* p, int lane, int n) {
        load_f32<A == kVector>(p, lane, A == kMasked ? n : kWarpElems, x);
    }
    template <Access A>
    __device__ __forceinline__ void arrange(long long, int) {}
    __device__ __forceinline__ Pair get(int i) const { return x[i]; }
};
template <> struct GradRaw<__nv_bfloat16> {
    uint32_t x[4], after;        // bf16 is the high half of a binary32: widening is a shift, exact
    template <Access A>
    __device__ __forceinline__ void load(const __nv_bfloat16* from, int lane, int n) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(from);
        if (A == kVector) {
            const uint4 r = __ldcs(reinterpret_cast<const uint4*>(p + 8 * lane));
            x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
        } else if (A == kRows) {
            // words of two; a row at an odd element begins in the word of the element before it and has 129 words
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            const uint32_t* words = reinterpret_cast<const uint32_t*>(at & ~static_cast<uintptr_t>(3));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __ldcs(words + lane + 32 * i);
            after = __ldcs(words + (at & 2 ? 128 : 0));          // without a branch, which would part the loads
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = lane + 64 * i;
                const uint32_t l = j < n ? __ldcs(p + j) : 0u, h = j + 32 < n ? __ldcs(p + j + 32) : 0u;
                x[i] = l | h << 16;
            }
        }
    }
    // kRows, an odd row: a pair's second element is in the next lane's word.
    template <Access A>
    __device__ __forceinline__ void arrange(long long at, int lane) {
        if (A != kRows || (at & 2) == 0) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t up = __shfl_down_sync(0xffffffffu, x[i], 1);
            const uint32_t row = __shfl_sync(0xffffffffu, i < 3 ? x[i + 1] : after, 0);
            x[i] = __byte_perm(x[i], lane == 31 ? row : up, 0x5432);
        }
    }
    __device__ __forceinline__ Pair get(int i) const {
        return pack(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
    }
};

// kRows' elements to memory (a multiple of eight elements from an aligned address), or to consecutive ones by way of 256
// floats of shared memory.
template <typename GT>
__device__ __forceinline__ void store_rows(float* p, int lane, const Pair (&x)[4]) {
    if (sizeof(GT) == 4) {
        store_f32<false>(p, lane, kWarpElems, x);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<Pair*>(p)[lane + 32 * i] = x[i];
    }
}
template <typename GT>
__device__ __forceinline__ void to_vector(float* buffer, int lane, Pair (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (sizeof(GT) == 4) {
            buffer[lane + 64 * i] = lo(x[i]);
            buffer[lane + 64 * i + 32] = hi(x[i]);
        } else {
            reinterpret_cast<Pair*>(buffer)[lane + 32 * i] = x[i];
        }
    }
    __syncwarp();
    const ulonglong2* q = reinterpret_cast<const ulonglong2*>(buffer) + 2 * lane;
    const ulonglong2 a = q[0], b = q[1];
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

// g = sum over the active workers of lambda_k g_k: products rounded to fp32, added in order within groups of four
// workers, the groups' sums added in order.  Chains stay short, two sums are all that is held, and a pair's product and
// sum cost what two FMAs do.  KU workers' loads at once; MANY: more than KU workers, in rounds.
template <int KU>
__device__ __forceinline__ void pointers_of(const Source& s, const long long* grads, int k0, long long (&from)[KU]) {
#pragma unroll
    for (int j = 0; j < KU; ++j) from[j] = k0 + j < s.K ? __ldg(grads + s.worker[k0 + j]) : 0;
}
template <typename GT, int KU, Access A>
__device__ __forceinline__ void load_round(const Source& s, const long long (&from)[KU], int k0, int offset, int lane, int n,
                                           GradRaw<GT> (&raw)[KU]) {
#pragma unroll
    for (int j = 0; j < KU; ++j)
        if (k0 + j < s.K) raw[j].template load<A>(reinterpret_cast<const GT*>(from[j]) + offset, lane, n);
}
// offset is a multiple of 256: a row is odd where its tensor is
template <typename GT, int KU, Access A>
__device__ __forceinline__ void arrange_round(const Source& s, const long long (&from)[KU], int k0, int lane, GradRaw<GT> (&raw)[KU]) {
#pragma unroll
    for (int j = 0; j < KU; ++j)
        if (A == kRows && k0 + j < s.K) raw[j].template arrange<A>(from[j], lane);
}
// Adds the round's groups to g; FIRST: g begins with them.
template <typename GT, int KU, bool FIRST>
__device__ __forceinline__ void weigh_round(const Source& s, const GradRaw<GT> (&raw)[KU], int k0, Pair (&g)[4]) {
#pragma unroll
    for (int j = 0; j < KU; j += 4) {
        if (j > 0 && k0 + j >= s.K) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Pair x = mul(s.lambda[k0 + j], raw[j].get(i));
#pragma unroll
            for (int l = j + 1; l < j + 4 && l < KU; ++l)
                if (k0 + l < s.K) x = add(mul(s.lambda[k0 + l], raw[l].get(i)), x, s.one);
            g[i] = FIRST && j == 0 ? x : add(x, g[i], s.one);
        }
    }
}
template <typename GT, int KU, bool MANY, Access A>
__device__ __forceinline__ void aggregate(const Source& s, const long long* grads, int offset, int lane, int n,
                                          Pair (&g)[4]) {
    GradRaw<GT> raw[KU];
    long long from[KU];
    if constexpr (!MANY) {
        pointers_of<KU>(s, grads, 0, from);
        load_round<GT, KU, A>(s, from, 0, offset, lane, n, raw);
        arrange_round<GT, KU, A>(s, from, 0, lane, raw);
        weigh_round<GT, KU, true>(s, raw, 0, g);
    } else {
        static_assert(KU % 4 == 0, "groups of four workers");
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = both(-0.0f);                  // adds nothing to anything
#pragma unroll 1
        for (int k0 = 0; k0 < s.K; k0 += KU) {
            pointers_of<KU>(s, grads, k0, from);
            load_round<GT, KU, A>(s, from, k0, offset, lane, n, raw);
            arrange_round<GT, KU, A>(s, from, k0, lane, raw);
            weigh_round<GT, KU, false>(s, raw, k0, g);
        }
    }
}

// Sum of the squares of a lane's eight aggregates, in fp64: a finite gradient beyond 1.8e19 or below 1e-19 has
// no fp32 square, and the clipping factor is then the correctly rounded one but for the sum's 2^-53.
__device__ __forceinline__ double sum_squares(const Pair (&g)[4]) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double a = lo(g[i]), b = hi(g[i]);
        s = fma(a, a, s);
        s = fma(b, b, s);
    }
    return s;
}

// ---- 8-bit moments --------------------------------------------------------------------------------
// 32 random bits for an element: two rounds of a 32 x 32 -> 64-bit multiply whose halves are folded together,
// keyed by the call's seed and step.  The multipliers are odd constants; 0xAC4C1B51 is one of Wellons' triple32 mixer,
// 0x85EBCA6B (the position's high word) one of Appleby's MurmurHash3 finalizer.  Bias and evenness of both halves are
// tested, not taken from them.
__device__ __forceinline__ uint32_t fold_multiply(uint32_t x, uint32_t m) {
    const uint64_t z = static_cast<uint64_t>(x) * m;
    return static_cast<uint32_t>(z >> 32) ^ static_cast<uint32_t>(z);
}
__device__ __forceinline__ uint32_t random_bits(uint32_t position_and_key, uint32_t key1) {
    return fold_multiply(fold_multiply(position_and_key, 0xAC4C1B51u) ^ key1, 0xD6E8FEB5u);
}

// e4m3 code of magnitude y in [0, 448], taken up to the next value with probability (distance below y) / (step).
// Scaled by 2^-120, the 8-bit type's exponents (subnormals included) are binary32's lowest ones, so the code is
// bits 20 .. 26 of the pattern and what is below them the distance.  Both are kept four bits further up, which also
// drops the sign: the code is then the word's top byte, and 16 random bits belong into bytes 1 and 2.
__device__ __forceinline__ uint32_t encode(float y_scaled, uint32_t chance) { return (__float_as_uint(y_scaled) << 4) + chance; }

// The random bits' byte 0 holds 128, so that the word is eight units in the last place (16 each) too high:
// y = |x| 2^-120 (448 / s) is off by less than five (an approximate reciprocal and two roundings), and where bytes 1
// and 2 of the word are zero, the word is within eight of a carry and cannot tell which code the exact y would get.
__device__ __forceinline__ uint32_t chance_low(uint32_t r) { return __byte_perm(r, 0x80u, 0x5104); }
__device__ __forceinline__ uint32_t chance_high(uint32_t r) { return __byte_perm(r, 0x80u, 0x5324); }
__device__ __forceinline__ uint32_t middle_bytes(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x6521); }
__device__ __forceinline__ bool unsure(uint32_t word) { return (word & 0x00ffff00u) == 0u; }

// The same word's top byte by fp64: q floor(y / q + r / 65536), q = 2^(max(exponent of y, -6) - 3).
__device__ __noinline__ uint32_t encode_exactly(float magnitude, float top, uint32_t chance) {
    const double y = static_cast<double>(magnitude) * 448.0 / static_cast<double>(top);
    int exponent = static_cast<int>(__double_as_longlong(y) >> 52) - 1023;
    exponent = max(exponent, -6);
    const double steps = floor(y * __longlong_as_double(static_cast<long long>(1023 + 3 - exponent) << 52) +
                               static_cast<double>(chance >> 8) * 0x1p-16);      // byte 0 dropped
    const float value = fminf(static_cast<float>(steps) * __uint_as_float(static_cast<uint32_t>(127 + exponent - 3) << 23), 448.0f);
    return __float_as_uint(value * 0x1p-120f) << 4;
}

// Block scale: a = max |x| over the warp's 256 elements, s = max(a, 2^-100).  A block with a value that is not
// finite gets a NaN scale and keep = 0 (codes are masked to zero).
struct BlockScale {
    float top, scale;
    uint32_t keep;
};
__device__ __forceinline__ BlockScale block_scale(float lane_top) {
    const uint32_t top = max(__reduce_max_sync(0xffffffffu, __float_as_uint(lane_top)), 0x0d800000u);   // bits of 2^-100
    const bool finite = top < 0x7f800000u;
    BlockScale r;
    r.top = __uint_as_float(top);
    r.scale = finite ? r.top * (1.0f / 448.0f) : __uint_as_float(0x7fffffffu);
    r.keep = finite ? 0xffffffffu : 0u;
    return r;
}
// max(|a|, |b|, |c|), NaN if one is
__device__ __forceinline__ float top_of(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float top_of(const Pair (&x)[4]) {
    return top_of(top_of(lo(x[0]), hi(x[0]), lo(x[1])), top_of(hi(x[1]), lo(x[2]), hi(x[2])), top_of(lo(x[3]), hi(x[3]), 0.0f));
}

// x 2^-120 (448 / s).  The factor is a normal number up to s = 2^14; above, x and s are brought down first (an x that
// this makes subnormal is far below the smallest code's distance to the next).
__device__ __forceinline__ void scale_down(const Pair (&x)[4], float s, Pair (&y)[4]) {
    if (s < 0x1p14f) {
        const Pair factor = both(reciprocal(s) * (448.0f * 0x1p-120f));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul(x[i], factor);
    } else {
        const Pair factor = both(reciprocal(s * 0x1p-114f) * (448.0f * 0x1p-120f));
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul(mul(x[i], both(0x1p-114f)), factor);
    }
}

// Codes element by element (lane + 32 i, those below n); aligned ones come through shared memory.
__device__ __forceinline__ void load_codes(const uint8_t* p, int lane, int n, uint32_t (&c)[2]) {
    c[0] = c[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (lane + 32 * i < n) c[i >> 2] |= static_cast<uint32_t>(__ldcs(p + lane + 32 * i)) << (8 * (i & 3));
}
__device__ __forceinline__ void decode(const uint32_t (&c)[2], float scale, Pair (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(c[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x[i] = mul(pack(f.x, f.y), both(scale));
    }
}

// Codes of eight moments: the words' top bytes.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
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
// One step of the optimizer on a lane's eight elements, given the aggregate.
template <bool CLIP>
__device__ __forceinline__ void update(const StepArgs& a, float factor, Pair decay, const Pair (&g)[4], Pair (&p)[4],
                                       Pair (&m)[4], Pair (&u)[4]) {
    const Pair one = a.src.one;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // every product and sum of the moments is rounded on its own: 8-bit codes depend on the last bit
        const Pair h = CLIP ? mul(g[i], both(factor)) : g[i];
        m[i] = add(mul(m[i], a.beta1), mul(h, a.one_minus_beta1), one);
        u[i] = add(mul(u[i], a.beta2), mul(mul(h, h), a.one_minus_beta2), one);
        const Pair d = mul_add(pack(root(lo(u[i])), root(hi(u[i]))), a.inv_sqrt_c2, a.eps);
        const Pair move = mul(m[i], pack(reciprocal(lo(d)), reciprocal(hi(d))));
        p[i] = mul_add(a.minus_step_size, move, mul(p[i], decay));
    }
}
__device__ __forceinline__ Pair decay_of(const StepArgs& a, const long long* rec) {
    return both(1.0f - a.lr * __uint_as_float(static_cast<uint32_t>(__ldg(rec + kRecDecay))));
}

template <bool ALIGNED>
__device__ __forceinline__ void store_copy(long long to, int offset, int lane, int n, const Pair (&p)[4]) {
    __nv_bfloat16* w = reinterpret_cast<__nv_bfloat16*>(to) + offset;
    if (ALIGNED) {
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(lo(p[i]), hi(p[i]));
            r[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        __stcs(reinterpret_cast<uint4*>(w + 8 * lane), make_uint4(r[0], r[1], r[2], r[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = lane + 64 * i;
            if (j < n) w[j] = __float2bfloat16_rn(lo(p[i]));
            if (j + 32 < n) w[j + 32] = __float2bfloat16_rn(hi(p[i]));
        }
    }
}

// Both moments of a block to 8 bits; scales by lane 0.  Elements beyond the block's end have zero moments and leave the
// maximum alone.
template <bool ALIGNED>
__device__ __forceinline__ void encode_moments(const StepArgs& a, float* first_scale, float* second_scale, long long position,
                                               int lane, const Pair (&m)[4], const Pair (&u)[4], uint32_t (&cm)[2],
                                               uint32_t (&cu)[2]) {
    const BlockScale sm = block_scale(top_of(m)), su = block_scale(top_of(u));
    Pair ym[4], yu[4];
    scale_down(m, sm.top, ym);
    scale_down(u, su.top, yu);
    // position is a multiple of 256: its high word is the whole block's, and the lane's index does not carry
    const uint32_t base = (static_cast<uint32_t>(position) + (ALIGNED ? 8 * lane : lane)) ^ a.key0;
    const uint32_t key1 = a.key1 ^ (static_cast<uint32_t>(position >> 32) * 0x85EBCA6Bu);
    uint32_t wm[8], wu[8], clear = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t r = random_bits(base ^ (ALIGNED ? j : 32 * j), key1);
        wm[j] = encode(j & 1 ? hi(ym[j >> 1]) : lo(ym[j >> 1]), chance_low(r));
        wu[j] = encode(j & 1 ? hi(yu[j >> 1]) : lo(yu[j >> 1]), chance_high(r));
        clear = __vminu2(clear, middle_bytes(wm[j], wu[j]));
    }
    if ((clear & 0xffffu) == 0u || clear < 0x10000u) {            // one lane in 4,000, with its sixteen codes
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = random_bits(base ^ (ALIGNED ? j : 32 * j), key1);
            const float xm = fabsf(j & 1 ? hi(m[j >> 1]) : lo(m[j >> 1])), xu = fabsf(j & 1 ? hi(u[j >> 1]) : lo(u[j >> 1]));
            if (unsure(wm[j])) wm[j] = encode_exactly(xm, sm.top, chance_low(r));
            if (unsure(wu[j])) wu[j] = encode_exactly(xu, su.top, chance_high(r));
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) wm[j] |= __float_as_uint(j & 1 ? hi(m[j >> 1]) : lo(m[j >> 1])) & 0x80000000u;
    cm[0] = top_bytes(wm[0], wm[1], wm[2], wm[3]) & sm.keep;
    cm[1] = top_bytes(wm[4], wm[5], wm[6], wm[7]) & sm.keep;
    cu[0] = top_bytes(wu[0], wu[1], wu[2], wu[3]);
    cu[1] = top_bytes(wu[4], wu[5], wu[6], wu[7]);
    // A second moment that is not zero is never held as zero: the next step divides by its root.  Codes are below
    // 128, so a byte is zero where subtracting one borrows into its top bit.
    if (((cu[0] - 0x01010101u) | (cu[1] - 0x01010101u)) & 0x80808080u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = j & 1 ? hi(u[j >> 1]) : lo(u[j >> 1]);
            const uint32_t least = x != 0.0f ? 1u << (8 * (j & 3)) : 0u;
            if ((cu[j >> 2] >> (8 * (j & 3)) & 0xffu) == 0u) cu[j >> 2] |= least;
        }
    }
    cu[0] &= su.keep;
    cu[1] &= su.keep;
    if (lane == 0) {
        *first_scale = sm.scale;
        *second_scale = su.scale;
    }
}

// A block straight from global memory to registers and back.  A: kVector; kRows (vectors but for the gradients, which
// go through `buffer`, 256 floats of shared memory); kMasked.
template <typename GT, int KU, bool MANY, bool STATE8, bool CLIP, bool NORM, Access A>
__device__ __forceinline__ void step_block(const StepArgs& a, const long long* rec, int offset, int lane, int n, float factor,
                                           float* buffer, double& sq) {
    constexpr bool ALIGNED = A != kMasked;
    float* param = reinterpret_cast<float*>(__ldg(rec + kRecParam)) + offset;
    Pair p[4], m[4], u[4], g[4];
    // sixteen workers' rows take more registers: their sum first, then the states (25M elements: 482 -> 298 us; fewer
    // workers lose by it, 4 fp32 ones 158 -> 171 us)
    constexpr bool kSumFirst = A == kRows && (KU == 16 || MANY);
    if (kSumFirst) aggregate<GT, KU, MANY, A>(a.src, rec + kRecGrads, offset, lane, n, g);
    load_f32<ALIGNED>(param, lane, n, p);
    const long long first = __ldg(rec + kRecFirst), second = __ldg(rec + kRecSecond);
    float *first_scale = nullptr, *second_scale = nullptr;
    if (STATE8) {
        first_scale = reinterpret_cast<float*>(__ldg(rec + kRecFirstScale)) + offset / kWarpElems;
        second_scale = reinterpret_cast<float*>(__ldg(rec + kRecSecondScale)) + offset / kWarpElems;
        uint32_t c[2];
        load_codes(reinterpret_cast<const uint8_t*>(first) + offset, lane, n, c);
        decode(c, *first_scale, m);
        load_codes(reinterpret_cast<const uint8_t*>(second) + offset, lane, n, c);
        decode(c, *second_scale, u);
    } else {
        load_f32<ALIGNED>(reinterpret_cast<const float*>(first) + offset, lane, n, m);
        load_f32<ALIGNED>(reinterpret_cast<const float*>(second) + offset, lane, n, u);
    }
    const long long position = __ldg(rec + kRecPosition) + offset;
    if (CLIP && a.src.staged)
        load_f32<ALIGNED>(a.src.staged + position, lane, n, g);
    else if (!kSumFirst)
        aggregate<GT, KU, MANY, A>(a.src, rec + kRecGrads, offset, lane, n, g);
    if (A == kRows) to_vector<GT>(buffer, lane, g);
    if (NORM) sq += sum_squares(g);
    update<CLIP>(a, factor, decay_of(a, rec), g, p, m, u);
    store_f32<ALIGNED>(param, lane, n, p);
    if (const long long copy = __ldg(rec + kRecCopy)) store_copy<ALIGNED>(copy, offset, lane, n, p);
    if (STATE8) {
        uint32_t cm[2], cu[2];
        encode_moments<ALIGNED>(a, first_scale, second_scale, position, lane, m, u, cm, cu);
        store_codes<ALIGNED>(reinterpret_cast<uint8_t*>(first) + offset, lane, n, cm);
        store_codes<ALIGNED>(reinterpret_cast<uint8_t*>(second) + offset, lane, n, cu);
    } else {
        store_f32<ALIGNED>(reinterpret_cast<float*>(first) + offset, lane, n, m);
        store_f32<ALIGNED>(reinterpret_cast<float*>(second) + offset, lane, n, u);
    }
}

// The same for a block off the vector grid or shorter than 256, kept out of the kernels' registers.
template <typename GT, bool STATE8, bool CLIP, bool NORM>
__device__ __noinline__ double step_block_slow(const StepArgs& a, const long long* rec, int offset, int lane, int n, float factor) {
    double sq = 0.0;
    step_block<GT, 4, true, STATE8, CLIP, NORM, kMasked>(a, rec, offset, lane, n, factor, nullptr, sq);
    return sq;
}

// Norm and clipping factor from the sum of squares: max_norm / norm where the norm is larger than max_norm, else 1
// (a NaN norm does not clip).
__device__ __forceinline__ void write_norm(double total, float* norm, float* factor, float max_norm) {
    const double root = sqrt(total);
    if (norm) *norm = static_cast<float>(root);
    if (factor) *factor = root > static_cast<double>(max_norm) ? static_cast<float>(max_norm / root) : 1.0f;
}

template <bool CLIP>
__device__ __forceinline__ float clip_factor(const StepArgs& a, int lane) {
    if (!CLIP) return 1.0f;
    if (a.partial_count == 0) return __ldcg(a.factor);
    double total = 0.0;
#pragma unroll 1
    for (int i = lane; i < a.partial_count; i += 256) {              // eight loads at once
        double x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + 32 * j < a.partial_count ? __ldcg(a.partials + i + 32 * j) : 0.0;
#pragma unroll
        for (int j = 0; j < 8; ++j) total += x[j];
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
    float factor;
    write_norm(total, blockIdx.x == 0 && threadIdx.x == 0 ? a.norm : nullptr, &factor, a.max_norm);
    return factor;
}

// A step's CTAs take the records in order, after a norm kernel in the opposite one: what that read or left last is
// still in the L2 (one fp32 gradient, 10M elements: 60.7 -> 59.0 us; 25M: 99.4 -> 98.4).
template <bool CLIP>
__device__ __forceinline__ const long long* record_of(const Source& s) {
    return s.recs + (CLIP ? s.records - 1 - blockIdx.x : blockIdx.x) * static_cast<long long>(s.stride);
}
// Asks the L2 for the record of a CTA of the next wave; the moments and gradients have streamed it out.
template <bool CLIP>
__device__ __forceinline__ void prefetch_record(const Source& s, const long long* rec) {
    if (blockIdx.x + kAhead < s.records && threadIdx.x < s.stride / 4)
        agg::prefetch_l2(rec + (CLIP ? -kAhead : kAhead) * s.stride + 4 * threadIdx.x);
}

// 32-bit moments: one CTA per record, one block per warp, all its loads in flight at once; sixteen warps (up to two
// workers 32) on an SM keep 64 KB and more on the way.
template <typename GT, int KU, bool MANY, bool CLIP, bool NORM>
__global__ void __launch_bounds__(kThreads, KU >= 4 ? 2 : 4) adamw_kernel(const __grid_constant__ StepArgs a) {
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const int lane = threadIdx.x & 31, offset = (threadIdx.x >> 5) * kWarpElems;
    const long long* rec = record_of<CLIP>(a.src);
    const long long cf = __ldg(rec + kRecCount);
    const int n = static_cast<int>(cf & 0xffffffffLL) - offset, flags = static_cast<int>(cf >> 32);
    const float factor = clip_factor<CLIP>(a, lane);
    double sq = 0.0;
    __shared__ __align__(16) float buffer[kSpan];
    if (n > 0) {
        if (flags & kStateAligned && n >= kWarpElems) {
            if (flags & kGradsAligned || (CLIP && a.src.staged))
                step_block<GT, KU, MANY, false, CLIP, NORM, kVector>(a, rec, offset, lane, kWarpElems, factor, nullptr, sq);
            else
                step_block<GT, KU, MANY, false, CLIP, NORM, kRows>(a, rec, offset, lane, kWarpElems, factor, buffer + offset, sq);
        } else
            sq = step_block_slow<GT, false, CLIP, NORM>(a, rec, offset, lane, min(n, kWarpElems), factor);
    }
    if (NORM) agg::store_norm_partial(a.partials, sq);
}

// ---- 8-bit moments: blocks through shared memory ------------------------------------------------------
// Fifty instructions an element keep a warp busy for as long as its loads take, and the registers that this needs
// leave few warps: with loads and arithmetic in turn the kernel reached 47 % of the DRAM's rate (issue slots 43 %
// busy).  So every warp copies ahead into shared memory of its own (cp.async, kept in order by commit groups; nobody
// waits for another warp) and computes on what has arrived.
// The unit is an item: a block's parameters, codes and scales, or up to 2 KB of its gradients (four bf16 or two fp32
// workers); one or two workers travel with the parameters.  Small items keep the amount in flight even: with 4 KB of
// gradients an item, 110M parameters and 8 bf16 workers took 623 us, with 2 KB 554.

__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A slot of the ring.  Parameters, codes, scales (padded to 16 bytes); a worker's row of gradients, with room for the
// piece by which a row off the 16-byte grid is longer.
constexpr int kSlotCodes = 4 * kWarpElems, kSlotScales = kSlotCodes + 2 * kWarpElems, kSlotState = kSlotScales + 16;
template <typename GT, int KI>
struct Ring {
    static constexpr bool kFused = KI <= 2;                                   // gradients behind the parameters, in one item
    static constexpr int kItem = kFused ? KI : 8 / static_cast<int>(sizeof(GT));                       // workers in an item
    static constexpr int kRow = static_cast<int>(sizeof(GT)) * kWarpElems, kLongRow = kRow + 16;     // off the grid
    static constexpr int kGrads = kFused ? kSlotState : 0;                    // where an item's gradients begin
    // whole lines of 128 bytes: with rows of fp32 16 bytes longer and slots as they came, 25M parameters and 4 workers
    // took 117 us instead of 113
    static constexpr int kUsed = kFused ? kSlotState + KI * kLongRow : kItem * kLongRow > kSlotState ? kItem * kLongRow : kSlotState;
    static constexpr int kSlot = (kUsed + 127) / 128 * 128;
    // two CTAs on an SM; with 104 KB instead of 88, a step behind a norm kernel was slower (25M elements: 98 -> 106 us)
    static constexpr int kMost = (88 << 10) / (kWarps * kSlot);
    static constexpr int kSlots = kMost < 6 ? kMost : 6;
    static constexpr int kBytes = kWarps * kSlots * kSlot;
};

// The first `have` bytes (none if it is negative) of BYTES, and zeros: the end of a buffer.
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, int have) {
    const int bytes = have < 0 ? 0 : have > BYTES ? BYTES : have;
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(BYTES), "r"(bytes) : "memory");
}

// One worker's 256 gradients to shared memory, in order; n < 256: and zeros behind the n-th.
template <bool FULL, typename GT>
__device__ __forceinline__ void copy_row(uint32_t to, const GT* from, int lane, int n) {
    constexpr int kSize = static_cast<int>(sizeof(GT)), kBytes = kSize * kWarpElems;
    const char* src = reinterpret_cast<const char*>(from);
#pragma unroll
    for (int i = 0; i < kBytes; i += 512) {
        const int at = i + 16 * lane;
        if (FULL) copy_async<16>(to + at, src + at);
        else copy_async<16>(to + at, src + at, kSize * n - at);
    }
}
// The same off the 16-byte grid: shared memory holds the row as far off it as global memory does, so that all but its
// first piece can be copied 16 bytes at a time.  The first goes by words, the last is cut behind the row; a bf16 row at
// an odd word half begins with the word that holds the element before it.  Rows copied by words to the grid: ragged 5M,
// three fp32 gradients, 30.0 us instead of 29.1; 25M, sixteen fp32 365 instead of 314, eight bf16 163 instead of 145.
template <bool FULL, typename GT>
__device__ __forceinline__ void copy_row_unaligned(uint32_t to, const GT* from, int lane, int n) {
    constexpr int kSize = static_cast<int>(sizeof(GT)), kBytes = kSize * kWarpElems;
    const uintptr_t address = reinterpret_cast<uintptr_t>(from);
    const int off = static_cast<int>(address & 15), have = kSize * n + off;
    const char* src = reinterpret_cast<const char*>(address - off);
    if (lane < 4 && 4 * lane + 4 > off) copy_async<4>(to + 4 * lane, src + 4 * lane, have - 4 * lane);
#pragma unroll
    for (int i = 16; i <= kBytes; i += 512) {
        const int at = i + 16 * lane;
        if (FULL && i + 512 < kBytes) copy_async<16>(to + at, src + at);
        else copy_async<16>(to + at, src + at, have - at);
    }
}

// A lane's elements of a slot.
__device__ __forceinline__ void read_pairs(const unsigned char* from, int lane, Pair (&x)[4]) {
    const ulonglong2* q = reinterpret_cast<const ulonglong2*>(from) + 2 * lane;
    const ulonglong2 a = q[0], b = q[1];
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
__device__ __forceinline__ void read_codes(const unsigned char* from, int lane, uint32_t (&x)[2]) {
    const uint2 r = reinterpret_cast<const uint2*>(from)[lane];
    x[0] = r.x; x[1] = r.y;
}
__device__ __forceinline__ void widen(const uint32_t* w, Pair (&x)[4]) {                      // bf16
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <typename GT>
__device__ __forceinline__ void read_row(const unsigned char* from, int lane, Pair (&x)[4]) {
    if constexpr (sizeof(GT) == 4) {
        read_pairs(from, lane, x);
    } else {
        const uint4 r = reinterpret_cast<const uint4*>(from)[lane];
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        widen(w, x);
    }
}
// A row that begins `off` bytes into its slot (the same for the whole warp).
template <typename GT>
__device__ __forceinline__ void read_row_at(const unsigned char* from, int lane, int off, Pair (&x)[4]) {
    constexpr int kWords = 2 * sizeof(GT);                                                   // of a lane
    uint32_t w[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords + 4; i += 4) {
        const uint4 r = reinterpret_cast<const uint4*>(from + 4 * kWords * lane)[i / 4];
        w[i] = r.x; w[i + 1] = r.y; w[i + 2] = r.z; w[i + 3] = r.w;
    }
    if (off & 8) {
#pragma unroll
        for (int i = 0; i < kWords + 2; ++i) w[i] = w[i + 2];
    }
    if (off & 4) {
#pragma unroll
        for (int i = 0; i < kWords + 1; ++i) w[i] = w[i + 1];
    }
    if constexpr (sizeof(GT) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    } else {
        if (off & 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], w[i + 1], 0x5432);
        }
        widen(w, x);
    }
}

// One kernel for each number KI of workers (1, 2, 4 or 8, taken for K in (KI / 2, KI]; MANY: more than that, in rounds).
template <typename GT, int KI, bool MANY, bool CLIP, bool NORM>
__global__ void __launch_bounds__(kThreads, 2) adamw8_kernel(const __grid_constant__ StepArgs a) {
    using R = Ring<GT, KI>;
    extern __shared__ __align__(16) unsigned char smem[];
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long* rec = record_of<CLIP>(a.src);
    const long long cf = __ldg(rec + kRecCount);
    const int count = static_cast<int>(cf & 0xffffffffLL);
    const bool grads_aligned = cf >> 32 & kGradsAligned || (CLIP && a.src.staged);
    const int K = a.src.K, items = R::kFused ? 1 : 1 + (K + R::kItem - 1) / R::kItem;         // of a block
    prefetch_record<CLIP>(a.src, rec);
    double sq = 0.0;

    // blocks warp, warp + 8, ... of the run; those of aligned tensors come through the ring
    const int mine = (count - warp * kWarpElems + kSpan - 1) / kSpan;                        // blocks that begin in the run
    const int blocks = cf >> 32 & kStateAligned ? mine : 0;
    const int whole = blocks - (blocks > 0 && warp * kWarpElems + (blocks - 1) * kSpan + kWarpElems > count);
    const unsigned char* slots = smem + warp * (R::kSlots * R::kSlot);
    const uint32_t ring = shared_address(slots);
    const char* params = reinterpret_cast<const char*>(__ldg(rec + kRecParam));
    const char* first = reinterpret_cast<const char*>(__ldg(rec + kRecFirst));
    const char* second = reinterpret_cast<const char*>(__ldg(rec + kRecSecond));
    const char* first_scale = reinterpret_cast<const char*>(__ldg(rec + kRecFirstScale));
    const char* second_scale = reinterpret_cast<const char*>(__ldg(rec + kRecSecondScale));
    const long long position = __ldg(rec + kRecPosition);
    // what a lane copies of every block, at the run's first element
    const char* my_params = params + 16 * lane;
    const char* my_codes = (lane < 16 ? first : second) + 16 * (lane & 15);
    const char* my_scale = lane == 0 ? first_scale : second_scale;
    // The gradients' pointers, worker by worker in the lanes: a shuffle fetches one, where a load for each copy would
    // put its latency into every item.
    const int other = lane + 32;
    long long from_low = lane < K ? __ldg(rec + kRecGrads + a.src.worker[lane]) : 0;
    const long long from_high = MANY && other < K ? __ldg(rec + kRecGrads + a.src.worker[other]) : 0;
    if (CLIP && a.src.staged) from_low = reinterpret_cast<long long>(a.src.staged + position);
    auto copy_item = [&](auto full, int offset, int item, uint32_t to) {
        constexpr bool kFull = decltype(full)::value;
        const int n = kFull ? kWarpElems : count - offset;
        if (R::kFused || item == 0) {
            if (kFull) {
                copy_async<16>(to + 16 * lane, my_params + 4 * offset);
                copy_async<16>(to + 512 + 16 * lane, my_params + 4 * offset + 512);
                copy_async<16>(to + kSlotCodes + 16 * lane, my_codes + offset);
            } else {
                copy_async<16>(to + 16 * lane, my_params + 4 * offset, 4 * n - 16 * lane);
                copy_async<16>(to + 512 + 16 * lane, my_params + 4 * offset + 512, 4 * n - 512 - 16 * lane);
                copy_async<16>(to + kSlotCodes + 16 * lane, my_codes + offset, n - 16 * (lane & 15));
            }
            if (lane < 2) copy_async<4>(to + kSlotScales + 4 * lane, my_scale + offset / (kWarpElems / 4));
        }
        if (R::kFused || item > 0) {
            const int k0 = R::kFused ? 0 : (item - 1) * R::kItem;
            auto row = [&](int j) {
                const int k = k0 + j;
                return reinterpret_cast<const GT*>(__shfl_sync(0xffffffffu, MANY && k >= 32 ? from_high : from_low, k & 31)) + offset;
            };
            if (kFull && grads_aligned) {
#pragma unroll
                for (int j = 0; j < R::kItem; ++j)
                    if (R::kFused || k0 + j < K) copy_row<true>(to + R::kGrads + j * R::kRow, row(j), lane, n);
            } else {
#pragma unroll 1
                for (int j = 0; j < R::kItem && (R::kFused || k0 + j < K); ++j) {
                    if (grads_aligned) copy_row<false>(to + R::kGrads + j * R::kRow, row(j), lane, n);
                    else copy_row_unaligned<kFull>(to + R::kGrads + j * R::kLongRow, row(j), lane, n);
                }
            }
        }
    };

    int next_offset = warp * kWarpElems, next_item = 0;                                       // the item to copy
    int left = whole * items, rest = (blocks - whole) * items;                               // of whole blocks, of a shorter one
    uint32_t to = ring;
    const unsigned char* from = slots;
    auto issue = [&]() {
        if (left > 0) {
            copy_item(std::true_type(), next_offset, next_item, to);
            --left;
            if (R::kFused || ++next_item == items) {
                next_item = 0;
                next_offset += kSpan;
            }
        } else if (rest > 0) {
            copy_item(std::false_type(), next_offset, next_item++, to);
            --rest;
        }
        copy_commit();                       // an empty group where nothing is left: the count of groups stays right
        to = to == ring + (R::kSlots - 1) * R::kSlot ? ring : to + R::kSlot;
    };
    auto arrive = [&]() {                    // the item at `from` is there, another one on its way
        issue();
        copy_wait<R::kSlots - 1>();
        __syncwarp();
    };
    auto release = [&]() {                   // everybody has read the slot before anybody's copy overwrites it
        __syncwarp();
        from = from == slots + (R::kSlots - 1) * R::kSlot ? slots : from + R::kSlot;
    };
#pragma unroll 1
    for (int i = 0; i < R::kSlots - 1; ++i) issue();

    const float factor = clip_factor<CLIP>(a, lane);
    const Pair decay = decay_of(a, rec);
    const long long copy = __ldg(rec + kRecCopy);
    int offset = warp * kWarpElems;
    // A block.  Whole ones with their rows on the grid, and off it, are loops of their own: tests for the others in the
    // first cost 3 to 6 %.
    auto do_block = [&](auto whole_block, auto on_grid) {
        constexpr bool kWhole = decltype(whole_block)::value, kOnGrid = decltype(on_grid)::value;
        Pair sum[4], part[4], p[4];
        uint32_t cm[2], cu[2];
        float2 scales;
        arrive();
        read_pairs(from, lane, p);
        read_codes(from + kSlotCodes, lane, cm);
        read_codes(from + kSlotCodes + kWarpElems, lane, cu);
        scales = *reinterpret_cast<const float2*>(from + kSlotScales);
        if (!R::kFused) release();
        if (MANY) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = both(-0.0f);                                // adds nothing to anything
        }
#pragma unroll 1
        for (int round = 0; round < (MANY ? K : 1); round += KI) {
#pragma unroll
            for (int chunk = 0; chunk < KI; chunk += R::kItem) {
                if (MANY ? round + chunk >= K : chunk > KI / 2 && chunk >= K) break;         // no such item
                if (!R::kFused) arrive();
#pragma unroll
                for (int j = 0; j < R::kItem; ++j) {
                    const int place = chunk + j, k = MANY ? round + place : place;
                    if (MANY ? k < K : place <= KI / 2 || place < K) {
                        Pair x[4];
                        if (kOnGrid || (!kWhole && grads_aligned)) {
                            read_row<GT>(from + R::kGrads + j * R::kRow, lane, x);
                        } else {
                            const long long at = __shfl_sync(0xffffffffu, MANY && k >= 32 ? from_high : from_low, k & 31);
                            read_row_at<GT>(from + R::kGrads + j * R::kLongRow, lane, static_cast<int>(at & 15), x);
                        }
                        const Pair w = KI == 1 ? 0ull : a.src.lambda[k];                     // a single weight is 1
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const Pair y = KI == 1 ? x[i] : mul(w, x[i]);
                            part[i] = place % 4 == 0 ? y : add(y, part[i], a.src.one);
                        }
                    }
                }
                release();
                // the group of four is complete, or its last workers are missing and so is the item after this one
                const int next = chunk + R::kItem;
                if (next % 4 == 0 || next >= KI || (MANY ? round + next : next) >= K) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = !MANY && chunk < 4 ? part[i] : add(part[i], sum[i], a.src.one);
                }
            }
        }
        if (NORM) sq += sum_squares(sum);
        Pair m[4], u[4];
        decode(cm, scales.x, m);
        decode(cu, scales.y, u);
        update<CLIP>(a, factor, decay, sum, p, m, u);
        float* param = reinterpret_cast<float*>(const_cast<char*>(params)) + offset;
        uint8_t* codes_m = reinterpret_cast<uint8_t*>(const_cast<char*>(first)) + offset;
        uint8_t* codes_u = reinterpret_cast<uint8_t*>(const_cast<char*>(second)) + offset;
        if (kWhole) {
            store_f32<true>(param, lane, kWarpElems, p);
            if (copy) store_copy<true>(copy, offset, lane, kWarpElems, p);
        }
        encode_moments<true>(a, reinterpret_cast<float*>(const_cast<char*>(first_scale)) + offset / kWarpElems,
                             reinterpret_cast<float*>(const_cast<char*>(second_scale)) + offset / kWarpElems, position + offset,
                             lane, m, u, cm, cu);
        if (kWhole) {
            store_codes<true>(codes_m, lane, kWarpElems, cm);
            store_codes<true>(codes_u, lane, kWarpElems, cu);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 8 * lane + i;
                if (j >= count - offset) break;
                const float x = i & 1 ? hi(p[i >> 1]) : lo(p[i >> 1]);
                param[j] = x;
                if (copy) reinterpret_cast<__nv_bfloat16*>(copy)[offset + j] = __float2bfloat16_rn(x);
                codes_m[j] = static_cast<uint8_t>(cm[i >> 2] >> (8 * (i & 3)));
                codes_u[j] = static_cast<uint8_t>(cu[i >> 2] >> (8 * (i & 3)));
            }
        }
    };
    int block = 0;
    if (grads_aligned) {
#pragma unroll 1
        for (; block < whole; ++block, offset += kSpan) do_block(std::true_type(), std::true_type());
    } else {
#pragma unroll 1
        for (; block < whole; ++block, offset += kSpan) do_block(std::true_type(), std::false_type());
    }
    for (; block < blocks; ++block, offset += kSpan) do_block(std::false_type(), std::false_type());
    // tensors off the grid
#pragma unroll 1
    for (; block < mine; ++block, offset += kSpan)
        sq += step_block_slow<GT, true, CLIP, NORM>(a, rec, offset, lane, min(count - offset, kWarpElems), factor);
    if (NORM) agg::store_norm_partial(a.partials, sq);
}

// ---- the norm of the weighted gradient ------------------------------------------------------------------
// Two CTAs of 128 threads share a record of norm_batch CTA steps of 256; all loads of a CTA are in flight at once (16 to
// 32 KB of gradients); with a staging buffer it also leaves the aggregates there, for the step that follows.
// LAST: the CTA that arrives last adds all partials, in order, which saves a launch; on grids of many waves the
// fence and the atomic at every CTA's end cost more than it, and a fold kernel follows instead.

// Blocks of a warp whose loads are in flight at once, by the registers that they take (32 to 64).
template <typename GT>
__host__ __device__ constexpr int norm_batch(int workers) {
    return sizeof(GT) == 4 ? (workers <= 1 ? 4 : workers <= 2 ? 2 : 1) : (workers <= 1 ? 8 : workers <= 2 ? 4 : workers <= 4 ? 2 : 1);
}

template <typename GT>
__device__ __noinline__ double norm_block_slow(const Source& s, const long long* grads, int offset, int lane, int n, float* staged) {
    Pair g[4];
    aggregate<GT, 4, true, kMasked>(s, grads, offset, lane, n, g);
    if (staged) store_f32<false>(staged, lane, n, g);
    return sum_squares(g);
}

// A warp's `whole` >= 1 blocks of a batch.  Where they may be fewer than a batch (FULL == false), the last one is loaded
// again in place of the missing and not counted: no branch parts the loads.
template <typename GT, int KU, bool MANY, Access A, bool FULL>
__device__ __forceinline__ double norm_blocks(const Source& s, const long long* rec, const long long (&from)[KU], int base,
                                              int whole, int lane, float* staged) {
    constexpr int kBatch = norm_batch<GT>(KU);
    double sq = 0.0;
    GradRaw<GT> raw[kBatch][KU];
    if (!MANY) {
#pragma unroll
        for (int e = 0; e < kBatch; ++e)
            load_round<GT, KU, A>(s, from, 0, base + (FULL ? e : min(e, whole - 1)) * kSpan, lane, kWarpElems, raw[e]);
    }
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
        const int offset = base + e * kSpan;
        if (!FULL && e >= whole) break;
        Pair g[4];
        if constexpr (MANY) {
            aggregate<GT, KU, true, A>(s, rec + kNormGrads, offset, lane, kWarpElems, g);
        } else {
            arrange_round<GT, KU, A>(s, from, 0, lane, raw[e]);
            weigh_round<GT, KU, true>(s, raw[e], 0, g);
        }
        if (staged) {
            if (A == kVector) store_f32<true>(staged + offset, lane, kWarpElems, g);
            else store_rows<GT>(staged + offset, lane, g);
        }
        sq += sum_squares(g);
    }
    return sq;
}

// The end of a tensor: fewer blocks than a batch, the last one shorter than 256.  Kept out of the kernel's registers.
template <typename GT, int KU, bool MANY>
__device__ __noinline__ double norm_end(const Source& s, const long long* rec, int base, int whole, int lane, int count, bool aligned,
                                        float* staged) {
    double sq = 0.0;
    long long from[KU];
    if (!MANY) pointers_of<KU>(s, rec + kNormGrads, 0, from);
    if (whole > 0) {
        if (aligned) sq = norm_blocks<GT, KU, MANY, kVector, false>(s, rec, from, base, whole, lane, staged);
        else sq = norm_blocks<GT, KU, MANY, kRows, false>(s, rec, from, base, whole, lane, staged);
    }
    const int end = base + whole * kSpan;
    if (end < count)
        sq += norm_block_slow<GT>(s, rec + kNormGrads, end, lane, count - end, staged ? staged + end : nullptr);
    return sq;
}

template <typename GT, int KU, bool MANY, bool LAST>
__global__ void __launch_bounds__(kNormThreads, KU * sizeof(GT) > 16 || MANY ? 4 : 6) grad_norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int kBatch = norm_batch<GT>(KU);
    __shared__ double smem[kWarps];
    __shared__ bool last;
    agg::griddep_launch_dependents();
    agg::griddep_wait();
    const int lane = threadIdx.x & 31;
    const int base = ((threadIdx.x + (blockIdx.x & 1) * kNormThreads) >> 5) * kWarpElems;
    const long long* rec = a.src.recs + (blockIdx.x >> 1) * static_cast<long long>(a.src.stride);
    const long long cf = __ldg(rec + kNormCount);
    const int count = static_cast<int>(cf & 0xffffffffLL);
    float* staged = a.src.staged ? a.src.staged + __ldg(rec + kNormPosition) : nullptr;
    // the pointers with the count, not behind the branch on it: one trip to memory before the gradients' own
    long long from[KU];
    if constexpr (!MANY) pointers_of<KU>(a.src, rec + kNormGrads, 0, from);
    // and the record of a CTA of the next wave to the L2, out of which the gradients have streamed it
    if ((blockIdx.x >> 1) + kAhead < a.src.records && threadIdx.x < a.src.stride / 4)
        agg::prefetch_l2(rec + kAhead * a.src.stride + 4 * threadIdx.x);
    double sq = 0.0;
    const int whole = (count - base - kWarpElems + kSpan) / kSpan;           // of 256
    const bool aligned = cf >> 32 & kGradsAligned;
    if (whole >= kBatch) {
        if (aligned) sq = norm_blocks<GT, KU, MANY, kVector, true>(a.src, rec, from, base, kBatch, lane, staged);
        else sq = norm_blocks<GT, KU, MANY, kRows, true>(a.src, rec, from, base, kBatch, lane, staged);
    } else if (base < count) {
        sq = norm_end<GT, KU, MANY>(a.src, rec, base, max(whole, 0), lane, count, aligned, staged);
    }

    const double mine = agg::block_sum(sq, smem);
    if (!LAST) {
        if (threadIdx.x == 0) a.partials[blockIdx.x] = mine;
        return;
    }
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = mine;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double acc = 0.0;
    for (unsigned int i = threadIdx.x; i < gridDim.x; i += kNormThreads) acc += __ldcg(a.partials + i);
    const double total = agg::block_sum(acc, smem);
    if (threadIdx.x != 0) return;
    *a.ticket = 0u;
    write_norm(total, a.norm, a.factor, a.max_norm);
}

// Folds partials: CTA c sums [c per, (c + 1) per); the last stage (one CTA, sums == NULL) writes the norm.
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
    if (sums) sums[blockIdx.x] = total;
    else write_norm(total, norm, factor, max_norm);
}

}  // namespace adamw
}  // namespace dynbatch
