// What follows a layer's product on the accumulator, 32 columns of a row per thread: bias, activation, residual, gating and
// its gradient, and what is kept for the backward pass.  All in fp32, two values per instruction where there is one for two.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "checkpoint8.cuh"
#include "dynbatch.h"

namespace dynbatch {
namespace lg {

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

// ------------------------------------------------------------------------------------------------ two floats
using Pair = unsigned long long;

__device__ __forceinline__ Pair pair(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void halves(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair both(float x) { return pair(x, x); }
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair add(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair mul_add(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// ------------------------------------------------------------------------------------------------ 32 values of a row
__device__ __forceinline__ bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

__device__ __forceinline__ void unpack2(uint32_t two, float& a, float& b) {
    a = __uint_as_float(two << 16);
    b = __uint_as_float(two & 0xFFFF0000u);
}
__device__ __forceinline__ Pair unpack_pair(uint32_t two) { return pair(__uint_as_float(two << 16), __uint_as_float(two & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ uint32_t pack_pair(Pair p) {
    float a, b;
    halves(p, a, b);
    return pack2(a, b);
}
// Accesses of 32 bytes: a thread has a row of its own, so a warp's access touches 32 lines, and the fewer accesses the better.
__device__ __forceinline__ void load32(const void* p, uint32_t* q) {
    unsigned long long x[4];
    asm volatile("ld.global.v4.b64 {%0,%1,%2,%3}, [%4];" : "=l"(x[0]), "=l"(x[1]), "=l"(x[2]), "=l"(x[3]) : "l"(p) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[2 * i] = static_cast<uint32_t>(x[i]);
        q[2 * i + 1] = static_cast<uint32_t>(x[i] >> 32);
    }
}
__device__ __forceinline__ void store32(void* p, const uint32_t* q) {
    unsigned long long x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = q[2 * i] | (static_cast<unsigned long long>(q[2 * i + 1]) << 32);
    asm volatile("st.global.v4.b64 [%0], {%1,%2,%3,%4};" ::"l"(p), "l"(x[0]), "l"(x[1]), "l"(x[2]), "l"(x[3]) : "memory");
}
__device__ __forceinline__ void load16(const void* p, uint32_t* q) {
    const uint4 x = *static_cast<const uint4*>(p);
    q[0] = x.x; q[1] = x.y; q[2] = x.z; q[3] = x.w;
}
__device__ __forceinline__ void store16(void* p, const uint32_t* q) { *static_cast<uint4*>(p) = make_uint4(q[0], q[1], q[2], q[3]); }

// BYTES bytes of a row, `valid` of them there (the rest zero), in units of `UNIT` bytes: the widest access that address
// and length allow.
template <int BYTES, class UNIT>
__device__ __forceinline__ void load_bytes(const UNIT* p, int valid, uint32_t (&q)[BYTES / 4]) {
    if (valid == BYTES / static_cast<int>(sizeof(UNIT)) && aligned_to(p, 16)) {
        if (aligned_to(p, 32)) {
#pragma unroll
            for (int i = 0; i < BYTES / 32; ++i) load32(reinterpret_cast<const char*>(p) + 32 * i, q + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) load16(reinterpret_cast<const char*>(p) + 16 * i, q + 4 * i);
        }
    } else if (valid == BYTES / static_cast<int>(sizeof(UNIT))) {
        // off the 16-byte grid: whole words from the first word boundary on, the bytes before and behind them one by one
        const unsigned char* b = reinterpret_cast<const unsigned char*>(p);
        const int lead = static_cast<int>((4 - (reinterpret_cast<uintptr_t>(p) & 3)) & 3);
        uint32_t head = 0, tail = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            if (j < lead) head |= static_cast<uint32_t>(b[j]) << (8 * (4 - lead + j));     // at the word's top
            if (lead && j < 4 - lead) tail |= static_cast<uint32_t>(b[BYTES - 4 + lead + j]) << (8 * j);
        }
        uint32_t before = head;
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) {
            uint32_t word = tail;
            if (i < BYTES / 4 - 1 || lead == 0) word = *reinterpret_cast<const uint32_t*>(b + lead + 4 * i);
            q[i] = lead ? __funnelshift_r(before, word, 8 * (4 - lead)) : word;
            before = word;
        }
    } else {
        constexpr int kPer = 4 / sizeof(UNIT);
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) {
            q[i] = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (i * kPer + j < valid) q[i] |= static_cast<uint32_t>(p[i * kPer + j]) << (8 * sizeof(UNIT) * j);
        }
    }
}
template <int BYTES, class UNIT>
__device__ __forceinline__ void store_bytes(UNIT* p, int valid, const uint32_t (&q)[BYTES / 4]) {
    if (valid == BYTES / static_cast<int>(sizeof(UNIT)) && aligned_to(p, 16)) {
        if (aligned_to(p, 32)) {
#pragma unroll
            for (int i = 0; i < BYTES / 32; ++i) store32(reinterpret_cast<char*>(p) + 32 * i, q + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) store16(reinterpret_cast<char*>(p) + 16 * i, q + 4 * i);
        }
    } else if (valid == BYTES / static_cast<int>(sizeof(UNIT))) {
        unsigned char* b = reinterpret_cast<unsigned char*>(p);
        const int lead = static_cast<int>((4 - (reinterpret_cast<uintptr_t>(p) & 3)) & 3);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            if (j < lead) b[j] = static_cast<unsigned char>(q[0] >> (8 * j));
            if (lead && j < 4 - lead) b[BYTES - 4 + lead + j] = static_cast<unsigned char>(q[BYTES / 4 - 1] >> (8 * (lead + j)));
        }
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i)
            if (i < BYTES / 4 - 1 || lead == 0)
                *reinterpret_cast<uint32_t*>(b + lead + 4 * i) = lead ? __funnelshift_r(q[i], q[i + 1 < BYTES / 4 ? i + 1 : i], 8 * lead) : q[i];
    } else {
        constexpr int kPer = 4 / sizeof(UNIT);
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i)
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (i * kPer + j < valid) p[i * kPer + j] = static_cast<UNIT>(q[i] >> (8 * sizeof(UNIT) * j));
    }
}
__device__ __forceinline__ void load_raw(const __nv_bfloat16* p, int n, uint32_t (&q)[16]) {
    load_bytes<64>(reinterpret_cast<const unsigned short*>(p), n, q);
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, int n, const Pair (&v)[16]) {
    uint32_t q[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = pack_pair(v[i]);
    store_bytes<64>(reinterpret_cast<unsigned short*>(p), n, q);
}
__device__ __forceinline__ void store_row(float* p, int n, const Pair (&v)[16]) {
    uint32_t q[kChunk];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        q[2 * i] = static_cast<uint32_t>(v[i]);
        q[2 * i + 1] = static_cast<uint32_t>(v[i] >> 32);
    }
    store_bytes<4 * kChunk>(reinterpret_cast<uint32_t*>(p), n, q);
}
// Values past the row's end are zero or NaN here (a product with the zeros that TMA reads there) and do not enter the scale.
__device__ __forceinline__ void keep_row(const Kept& k, int e4m3, long long row, int col, int N, int n, const Pair (&x)[16]) {
    if (!e4m3) {
        store_row(static_cast<__nv_bfloat16*>(k.data) + row * N + col, n, x);
        return;
    }
    float top = 0.f;                                           // maxima pass NaN over
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float a, b;
        halves(x[i], a, b);
        top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
    }
    uint32_t byte = ck8::scale_byte(top);
    uint32_t c[8];
    if (byte < ck8::kTopByte) {                                // and so top is finite
        const Pair inverse = both(ck8::scale_inverse(byte));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y[4];
            halves(mul(x[2 * i], inverse), y[0], y[1]);
            halves(mul(x[2 * i + 1], inverse), y[2], y[3]);
            c[i] = ck8::codes_of_finite(y[0], y[1], y[2], y[3]);
        }
    } else {
        top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float a, b;
            halves(x[i], a, b);
            top = fmaxf(top, fmaxf(ck8::finite_magnitude(a), ck8::finite_magnitude(b)));
        }
        byte = ck8::scale_byte(top);
        const float inverse = ck8::scale_inverse(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y[4];
            halves(x[2 * i], y[0], y[1]);
            halves(x[2 * i + 1], y[2], y[3]);
            c[i] = ck8::codes4(y[0], y[1], y[2], y[3], inverse, byte);
        }
    }
    k.scale[row * ((N + kChunk - 1) / kChunk) + col / kChunk] = static_cast<uint8_t>(byte);
    store_bytes<32>(static_cast<uint8_t*>(k.data) + row * N + col, n, c);
}
// A kept row as it lies in memory (16 words of bf16, or 8 of codes and the scale), fetched before it is needed.
struct RawRow {
    uint32_t q[16];
    uint32_t scale;
};
__device__ __forceinline__ void fetch_row(const Kept& k, int e4m3, long long row, int col, int N, int n, RawRow& r) {
    if (!e4m3) {
        load_raw(static_cast<const __nv_bfloat16*>(k.data) + row * N + col, n, r.q);
        return;
    }
    uint32_t c[8];
    load_bytes<32>(static_cast<const uint8_t*>(k.data) + row * N + col, n, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.q[i] = c[i];
    r.scale = k.scale[row * ((N + kChunk - 1) / kChunk) + col / kChunk];
}

// ------------------------------------------------------------------------------------------------ eight values of a row
// As loaded, so that a load under way holds no more registers than it has bytes.
template <class T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 q;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
        if (n == 8 && aligned_to(p, 16)) {
            q = *reinterpret_cast<const uint4*>(p);
        } else {
            uint32_t w[4];
            const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = (2 * j < n ? u[2 * j] : 0u) | (2 * j + 1 < n ? static_cast<uint32_t>(u[2 * j + 1]) << 16 : 0u);
            q = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ __forceinline__ void values(Pair (&v)[4]) const {
        v[0] = unpack_pair(q.x); v[1] = unpack_pair(q.y);
        v[2] = unpack_pair(q.z); v[3] = unpack_pair(q.w);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        unpack2(q.x, v[0], v[1]); unpack2(q.y, v[2], v[3]);
        unpack2(q.z, v[4], v[5]); unpack2(q.w, v[6], v[7]);
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p, int n) {
        if (n == 8 && aligned_to(p, 16)) {
            a = *reinterpret_cast<const float4*>(p);
            b = *(reinterpret_cast<const float4*>(p) + 1);
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.f;
            a = make_float4(v[0], v[1], v[2], v[3]);
            b = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
// The same for codes of a checkpoint.
struct Codes8 {
    uint2 q;
    __device__ __forceinline__ void load(const uint8_t* p, int n) {
        if (n == 8 && aligned_to(p, 8)) {
            q = *reinterpret_cast<const uint2*>(p);
        } else {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) w[j / 4] |= static_cast<uint32_t>(p[j]) << (8 * (j % 4));
            q = make_uint2(w[0], w[1]);
        }
    }
    __device__ __forceinline__ void values(uint32_t scale_byte, Pair (&v)[4]) const {
        const Pair scale = both(ck8::scale_value(scale_byte));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 t = ck8::values2((j < 2 ? q.x : q.y) >> (16 * (j % 2)));
            v[j] = mul(pair(t.x, t.y), scale);
        }
    }
};

// ------------------------------------------------------------------------------------------------ activations
// silu(z) = z s, s = 1 / (1 + e^-z);  gelu(z) = z P(z), P the normal distribution function.  The approximate exponential of v
// is off by about 2^-23 (1 + |v|), the reciprocal by 2^-23, relative, of a value that is rounded to 2^-9; arguments and results
// below 2^-126 count as 0.
// P by formula 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions: for x >= 0
//     erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) e^(-x^2),  t = 1 / (1 + 0.3275911 x),  off by at most 1.5e-7
// (relative to it 5e-4 at z = -4, 1.6e-3 at -5, 3.6e-3 at -6, where half a bf16 step is 3.9e-3 and gelu -6e-9),
// with x = |z| / sqrt(2): P is erfc / 2 below zero and 1 - erfc / 2 above, so gelu = max(z, 0) - |z| erfc / 2.  Two
// special-function instructions, and the e^(-z^2 / 2) is the one that the slope needs.  With erff the epilogue, not the
// products, set the time of a 1024-deep layer (8191 x 1024 to 4096: 92 us).
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2e = 1.44269504f;
constexpr Pair kSigns = 0x8000000080000000ull;
// Four pairs at a time, step by step: an epilogue warp has its scheduler almost to itself, and a chain of twenty dependent
// instructions, one pair after the other, left it idle for most of their latencies.
constexpr int kBatch = 4;
using Batch = Pair[kBatch];
#define DB_EACH _Pragma("unroll") for (int i = 0; i < kBatch; ++i)
__device__ __forceinline__ void exp2_batch(Batch& x) {
    DB_EACH {
        float a, b;
        halves(x[i], a, b);
        x[i] = pair(exp2_fast(a), exp2_fast(b));
    }
}
__device__ __forceinline__ void reciprocal_batch(Batch& x) {
    DB_EACH {
        float a, b;
        halves(x[i], a, b);
        x[i] = pair(reciprocal_fast(a), reciprocal_fast(b));
    }
}
__device__ __forceinline__ void sigmoid(const Batch& z, Batch& s) {
    DB_EACH s[i] = mul(z[i], both(-kLog2e));
    exp2_batch(s);
    DB_EACH s[i] = add(s[i], both(1.f));
    reciprocal_batch(s);
}
__device__ __forceinline__ Pair magnitude(Pair z) { return z & ~kSigns; }
// -min(|z|, the largest finite value): an infinity times a tail of zero is to be zero; a NaN stays one
__device__ __forceinline__ Pair minus_finite_magnitude(Pair z) {
    float a, b;
    halves(magnitude(z), a, b);
    asm("min.NaN.f32 %0, %0, 0f7F7FFFFF;" : "+f"(a));
    asm("min.NaN.f32 %0, %0, 0f7F7FFFFF;" : "+f"(b));
    return pair(-a, -b);
}
__device__ __forceinline__ Pair positive_part(Pair z) {       // a NaN stays one
    float a, b;
    halves(z, a, b);
    return pair(a < 0.f ? 0.f : a, b < 0.f ? 0.f : b);
}
// bell = e^(-z^2 / 2), tail = erfc(|z| / sqrt(2)) / 2
__device__ __forceinline__ void normal_tail(const Batch& z, Batch& bell, Batch& tail) {
    Batch t;
    DB_EACH t[i] = mul_add(magnitude(z[i]), both(0.23164190f), both(1.f));   // 0.3275911 / sqrt(2)
    DB_EACH bell[i] = mul(mul(z[i], both(-0.5f * kLog2e)), z[i]);
    reciprocal_batch(t);
    exp2_batch(bell);
    DB_EACH tail[i] = mul_add(both(0.5f * 1.061405429f), t[i], both(-0.5f * 1.453152027f));
    DB_EACH tail[i] = mul_add(tail[i], t[i], both(0.5f * 1.421413741f));
    DB_EACH tail[i] = mul_add(tail[i], t[i], both(-0.5f * 0.284496736f));
    DB_EACH tail[i] = mul_add(tail[i], t[i], both(0.5f * 0.254829592f));
    DB_EACH t[i] = mul(t[i], bell[i]);
    DB_EACH tail[i] = mul(tail[i], t[i]);
}
template <int ACT>
__device__ __forceinline__ void act_batch(Batch& z) {
    if (ACT == DB_ACT_SILU) {
        Batch s;
        sigmoid(z, s);
        DB_EACH z[i] = mul(z[i], s[i]);
    } else if (ACT == DB_ACT_GELU) {
        Batch bell, tail;
        normal_tail(z, bell, tail);
        DB_EACH z[i] = mul_add(minus_finite_magnitude(z[i]), tail[i], positive_part(z[i]));
    } else if (ACT == DB_ACT_RELU) {
        DB_EACH z[i] = positive_part(z[i]);
    }
}
template <int ACT>
__device__ __forceinline__ void act_batch_slope(const Batch& z, Batch& value, Batch& slope) {
    if (ACT == DB_ACT_SILU) {
        Batch s;
        sigmoid(z, s);
        DB_EACH value[i] = mul(z[i], s[i]);
        DB_EACH slope[i] = mul_add(s[i], both(-1.f), both(1.f));
        DB_EACH slope[i] = mul_add(value[i], slope[i], s[i]);
    } else if (ACT == DB_ACT_GELU) {
        Batch bell, tail;
        normal_tail(z, bell, tail);
        DB_EACH value[i] = mul_add(minus_finite_magnitude(z[i]), tail[i], positive_part(z[i]));
        // P(z) - 1/2 has z's sign and the magnitude 1/2 - tail
        DB_EACH slope[i] = mul_add(tail[i], both(-1.f), both(0.5f)) ^ (z[i] & kSigns);
        DB_EACH slope[i] = add(slope[i], both(0.5f));
        DB_EACH tail[i] = mul(z[i], both(0.39894228f));
        DB_EACH slope[i] = mul_add(tail[i], bell[i], slope[i]);
    } else if (ACT == DB_ACT_RELU) {
        DB_EACH {
            value[i] = positive_part(z[i]);
            float a, b;
            halves(z[i], a, b);
            slope[i] = pair(a <= 0.f ? 0.f : 1.f, b <= 0.f ? 0.f : 1.f);
        }
    } else {
        DB_EACH {
            value[i] = z[i];
            slope[i] = both(1.f);
        }
    }
}
// The branch on the activation is taken once for a row, not for each value.
template <int ACT>
__device__ __forceinline__ void act_row(Pair (&v)[16]) {
#pragma unroll
    for (int j = 0; j < 16; j += kBatch) {
        Batch b;
        DB_EACH b[i] = v[j + i];
        act_batch<ACT>(b);
        DB_EACH v[j + i] = b[i];
    }
}
__device__ __forceinline__ void act_row(Pair (&v)[16], int act) {
    if (act == DB_ACT_SILU) act_row<DB_ACT_SILU>(v);
    else if (act == DB_ACT_GELU) act_row<DB_ACT_GELU>(v);
    else if (act == DB_ACT_RELU) act_row<DB_ACT_RELU>(v);
}
// Sixteen columns at a time, stored as they are done, so that few results wait in registers.
template <int ACT, bool E4M3>
__device__ __forceinline__ void gated_grad_row(const Pair (&dh)[16], const RawRow& gate, const RawRow& up, __nv_bfloat16* d_gate,
                                               __nv_bfloat16* d_up, __nv_bfloat16* h, int n) {
    const Pair gate_scale = both(E4M3 ? ck8::scale_value(gate.scale) : 1.f), up_scale = both(E4M3 ? ck8::scale_value(up.scale) : 1.f);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t qg[8], qu[8], qh[8];
#pragma unroll
        for (int j = 0; j < 8; j += kBatch) {
            Batch z, u, a, s;
            DB_EACH {
                const int w = 8 * half + j + i;
                if (E4M3) {
                    const float2 x = ck8::values2(gate.q[w / 2] >> (16 * (w % 2))), y = ck8::values2(up.q[w / 2] >> (16 * (w % 2)));
                    z[i] = mul(pair(x.x, x.y), gate_scale);
                    u[i] = mul(pair(y.x, y.y), up_scale);
                } else {
                    z[i] = unpack_pair(gate.q[w]);
                    u[i] = unpack_pair(up.q[w]);
                }
            }
            act_batch_slope<ACT>(z, a, s);
            DB_EACH qh[j + i] = pack_pair(mul(a[i], u[i]));
            DB_EACH qu[j + i] = pack_pair(mul(dh[8 * half + j + i], a[i]));
            DB_EACH s[i] = mul(s[i], u[i]);
            DB_EACH qg[j + i] = pack_pair(mul(dh[8 * half + j + i], s[i]));
        }
        const int valid = min(16, n - 16 * half);
        if (valid > 0) {
            store_bytes<32>(reinterpret_cast<unsigned short*>(d_gate) + 16 * half, valid, qg);
            store_bytes<32>(reinterpret_cast<unsigned short*>(d_up) + 16 * half, valid, qu);
            store_bytes<32>(reinterpret_cast<unsigned short*>(h) + 16 * half, valid, qh);
        }
    }
}
template <bool E4M3>
__device__ __forceinline__ void gated_grad_row(int act, const Pair (&dh)[16], const RawRow& gate, const RawRow& up, __nv_bfloat16* d_gate,
                                               __nv_bfloat16* d_up, __nv_bfloat16* h, int n) {
    if (act == DB_ACT_SILU) gated_grad_row<DB_ACT_SILU, E4M3>(dh, gate, up, d_gate, d_up, h, n);
    else if (act == DB_ACT_GELU) gated_grad_row<DB_ACT_GELU, E4M3>(dh, gate, up, d_gate, d_up, h, n);
    else if (act == DB_ACT_RELU) gated_grad_row<DB_ACT_RELU, E4M3>(dh, gate, up, d_gate, d_up, h, n);
    else gated_grad_row<DB_ACT_NONE, E4M3>(dh, gate, up, d_gate, d_up, h, n);
}

// ------------------------------------------------------------------------------------------------ the epilogue of a row
// What the epilogue of 32 columns reads.
template <int EPI>
struct Fetched {
    uint32_t bias[16], addend[16];
};
template <>
struct Fetched<kEpiGated> {};
template <>
struct Fetched<kEpiGatedGrad> {
    RawRow gate, up;
};
template <int EPI>
__device__ __forceinline__ void epilogue_fetch(const EpilogueArgs& e, long long row, int col, int N, Fetched<EPI>& f) {
    const int n = min(kChunk, N - col);
    if constexpr (EPI == kEpiStore) {
        if (e.bias) load_raw(e.bias + col, n, f.bias);
        if (e.addend) load_raw(e.addend + row * e.addend_pitch + col, n, f.addend);
    } else if constexpr (EPI == kEpiGatedGrad) {
        fetch_row(e.kept[0], e.kept_e4m3, row, col, N, n, f.gate);
        fetch_row(e.kept[1], e.kept_e4m3, row, col, N, n, f.up);
    }
}
// Columns col (a multiple of 32) to col + 32, but not past N: v the accumulator (kEpiGated: gate's), u up's.
template <int EPI>
__device__ __forceinline__ void epilogue_row(const EpilogueArgs& e, long long row, int col, int N, const Fetched<EPI>& f, Pair (&v)[16],
                                             Pair (&u)[16]) {
    const int n = min(kChunk, N - col);
    if constexpr (EPI == kEpiStore) {
        if (e.bias) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = add(v[i], unpack_pair(f.bias[i]));
        }
        if (e.kept[0].data) keep_row(e.kept[0], e.kept_e4m3, row, col, N, n, v);
        act_row(v, e.act);
        if (e.addend) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = add(v[i], unpack_pair(f.addend[i]));
        }
        if (e.out_f32) store_row(static_cast<float*>(e.out) + row * e.out_pitch + col, n, v);
        else store_row(static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col, n, v);
    } else if constexpr (EPI == kEpiGated) {
        if (e.kept[0].data) {
            keep_row(e.kept[0], e.kept_e4m3, row, col, N, n, v);
            keep_row(e.kept[1], e.kept_e4m3, row, col, N, n, u);
        }
        act_row(v, e.act);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = mul(v[i], u[i]);
        store_row(static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col, n, v);
    } else {
        __nv_bfloat16* d_gate = e.d_gate + row * e.d_pitch + col;
        __nv_bfloat16* d_up = e.d_up + row * e.d_pitch + col;
        __nv_bfloat16* h = static_cast<__nv_bfloat16*>(e.out) + row * e.out_pitch + col;
        if (e.kept_e4m3) gated_grad_row<true>(e.act, v, f.gate, f.up, d_gate, d_up, h, n);
        else gated_grad_row<false>(e.act, v, f.gate, f.up, d_gate, d_up, h, n);
    }
}

#undef DB_EACH

}  // namespace lg
}  // namespace dynbatch
