// The bf16 matrix product of the layers (sm_100a, tcgen05), with what follows it done on the accumulator:
//     acc(m, n) = sum_k A(m, k) * B(n, k)          fp32 in tensor memory, operands bf16 by TMA
// Either operand may have the reduction index or the output index as its contiguous one, so that a layer's three
// products (y = x W, dx = dz W^T, dW = x^T dz) read x, W and dz from where they lie, W stored [in, out].
//
// One persistent CTA (or pair of CTAs) per SM (pair) walks the output tiles:
//   warp 0   copies 64-deep operand blocks into a ring of shared-memory stages by TMA
//   warp 1   owns the tensor memory and issues four tcgen05.mma a stage (of the pair's first CTA alone)
//            Both walk their loops as whole warps, one elected lane issues: the operands of the instructions are then
//            known to be uniform.  With one lane walking alone a 64-deep block took 0.32 us instead of 0.22.
//   the others take the finished accumulator out of tensor memory, 32 columns of a row per thread, apply the epilogue
//            and store; two accumulators, so that this runs under the next tile's products.
// A pair (cta_group::2) computes 256 rows x BN columns: each CTA holds its own 128 rows of A and half of B's, and the
// tensor cores of both read both halves, so an operand byte in shared memory serves twice as many products.
// Copies that serve a pair signal the first CTA's barrier; no multicast copies are used.
//
// Bound by the tensor cores where there are tiles for all pairs and the epilogue is plain: 16384 x 2048 x 2048, y 93 us,
// dx 89, dW 97 (64 tiles on 74 pairs), the tensor pipe 85 to 90 % active.  1024-deep products with more to do for each
// column are bound by the epilogue: 8191 x 1024 x 4096 48 us as it is, 55 with gelu, 59 with bias and gelu.  Its loads and
// stores are 32 bytes of a row for each thread, and the load/store unit takes each row as an access of its own.  Single CTAs
// start and end 1 us sooner than pairs; a first block costs them 4.7 us from the predecessor's end to their own, each further
// one 0.2.
//
// Every wait is bounded (2 s): whoever gives up sets the call's status word and its CTA's flag, all roles stop, copies
// and products under way are waited for (again with a limit), tensor memory is freed and the kernel returns.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "layer_epilogue.cuh"
#include "tc_gemm.cuh"

namespace dynbatch {
namespace lg {

constexpr int kRows = 128;             // rows of A a CTA holds = its tensor-memory lanes
constexpr int kBlockK = 64;            // bf16 in a 128-byte swizzled row
constexpr int kMaxProblems = 3;

struct Problem {
    CUtensorMap a[2], b[2];      // the reduction's two sources; kEpiGated: b[0] gate's and b[1] up's weights
    int M, N;                    // output rows and columns
    int blocks0, blocks;         // 64-deep blocks of the first source, and of both
    int m_tiles, n_tiles;
    long long partial;           // first float of this problem's partial sums
    EpilogueArgs e;
};

// Column sums to be finished on the side: out[c] = sum over i of sums[i][c], i ascending.
struct BiasFold {
    const float* sums = nullptr;        // [slabs][pitch]; nullptr: none
    long long pitch = 0;
    int slabs = 0, cols = 0, out_f32 = 0;
    void* out = nullptr;
};
// 32 columns a warp
__device__ __forceinline__ void fold_bias(const BiasFold& f, long long warp, long long warps, int lane) {
    for (long long c = warp * 32 + lane; c < f.cols; c += warps * 32) {
        float s = 0.f;
#pragma unroll 8
        for (int i = 0; i < f.slabs; ++i) s += f.sums[i * f.pitch + c];
        if (f.out_f32) static_cast<float*>(f.out)[c] = s;
        else static_cast<__nv_bfloat16*>(f.out)[c] = __float2bfloat16_rn(s);
    }
}

struct GemmArgs {
    Problem p[kMaxProblems];
    int tile_start[kMaxProblems + 1];   // first tile of a problem, and their number; a tile for each split
    int problems;
    int splits, blocks_per_split;       // splits > 1: the reduction is cut into pieces, whose fp32 sums combine_kernel joins
    float* partials;                    // [problem][split][gate, up][M][columns rounded up to 32]
    int* status;
    int clear_status;                   // the first CTA zeroes *status
    BiasFold bias;                      // kEpiStore: done by the epilogue's warps while they have no accumulator yet
};

// ------------------------------------------------------------------------------------------------ PTX wrappers
// Instructions marked .aligned want all lanes of the warp at the same instruction.  Code that lanes leave and rejoin (rows past
// the end, a row's own alignment) may stand before any of them, so each wrapper converges its warp itself.
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t columns) {
    __syncwarp();
    if (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tc::tmem_alloc(slot, columns);
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t columns) {
    __syncwarp();
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else tc::tmem_dealloc(base, columns);
}
// 32 columns of the warp's 32 rows of an accumulator, a row for each lane.
__device__ __forceinline__ void load_accumulator(uint32_t at, uint32_t (&raw)[32]) {
    __syncwarp();
    tc::tmem_load32(at, raw);
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
// The same, in this CTA alone: what gives up must leave nothing on its way to the other CTA, which may have left by then.
template <int CG>
__device__ __forceinline__ void mma_commit_here(uint64_t* bar) {
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(tc::smem_u32(bar)) : "memory");
    else
        tc::mma_commit(bar);
}
// A whole warp's bounded wait.  Lanes that poll on their own may differ where the limit runs out or the other warps give up, and
// those that went on would wait at the next full-warp instruction for those that left: all go on, or all leave.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status, int code) {
    return __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar, parity, abort_flag, status, code));
}
// True in one lane of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one() {
    uint32_t mine;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(mine));
    return mine != 0;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of the same shared-memory word in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first_cta(const void* p) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(0));
    return a;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    // no wider release than the default: it would wait for the warp's stores, which nobody here reads
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(tc::smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map, bool used) {
    if (used) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
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
    // A pair's CTA has an SM to itself and 192 KB of stages (6 of 32 KB, 8 of 24).  Two single CTAs share an SM, 96 KB each: one
    // works on its accumulator or starts up while the other's products run, a successor's among them.
    static constexpr int kCtas = CG == 2 ? 1 : 2;
    static constexpr int kStages = 196608 / kCtas / kStageBytes;
    static constexpr int kSmemBytes = kStages * kStageBytes + 1024;
    static constexpr int kEpilogueWarps = CG == 2 ? 8 : 4;   // two (one) per tensor-memory lane quarter, each its share of the columns
    static constexpr int kThreads = 64 + 32 * kEpilogueWarps;
    static constexpr uint32_t kTmemColumns = 2 * BN;         // two accumulators
    static_assert(kCtas * kTmemColumns <= 512 && (kTmemColumns & (kTmemColumns - 1)) == 0 && kTmemColumns >= 32, "a power of two up to 512");
    static_assert(kBRows >= 64 && BN % 64 == 0, "whole blocks of 64 output indices");
    static_assert(kCtas * (kSmemBytes + 1536) <= 233472, "228 KB with the barriers and what the system takes for each CTA");
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
__global__ void __launch_bounds__(Shape<CG, BN>::kThreads, Shape<CG, BN>::kCtas)
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
            tc::mbar_init(&taken_bar[i], CG * S::kEpilogueWarps);
        }
        tc::mbar_init(&drain_bar, 1);
        tc::fence_barrier_init();
    }
    if (warp == 0 && lane < 2) {
        const bool second = EPI == kEpiGated || g.p[0].blocks > g.p[0].blocks0;
        prefetch_map(lane == 0 ? &g.p[0].a[0] : &g.p[0].b[0], true);
        prefetch_map(lane == 0 ? &g.p[0].a[1] : &g.p[0].b[1], lane == 0 ? g.p[0].blocks > g.p[0].blocks0 : second);
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
        int stage = 0, it = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int t = worker; t < total && ok; t += workers) {
            const Tile tile = decode(g, t);
            const Problem& p = g.p[tile.problem];
            int k, k_end;
            k_range(g, tile, k, k_end);
            const int blocks0 = p.blocks0;
            const int m0 = tile.m * S::kTileM + static_cast<int>(rank) * kRows;
            // what this CTA holds of B: gated, a pair's CTAs take one weight each, a single CTA half of both
            const int n0 = tile.n * kTileN + (EPI == kEpiGated ? 0 : static_cast<int>(rank) * S::kBRows);
            for (; k < k_end; ++k, ++it) {
                if (!(ok = warp_wait(&empty_bar[stage], phase ^ 1, &abort_flag, g.status, 0x301))) break;
                if (elect_one()) {
                    const uint32_t bar = CG == 2 ? in_first_cta(&full_bar[stage]) : tc::smem_u32(&full_bar[stage]);
                    if (rank == 0) expect_tx(&full_bar[stage], CG * S::kStageBytes);
                    const int source = k >= blocks0;
                    const int k0 = (source ? k - blocks0 : k) * kBlockK;
                    const uint32_t a = tc::smem_u32(tiles + stage * S::kStageBytes), b = a + S::kABytes;
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
                __syncwarp();
                if (++stage == S::kStages) { stage = 0; phase ^= 1; }
            }
        }
        // every product that reads this CTA's stages has finished, and its arrival has reached this CTA
        for (int i = 0; i < S::kStages && ok && i < it; ++i) {
            if (--stage < 0) { stage = S::kStages - 1; phase ^= 1; }
            ok = warp_wait(&empty_bar[stage], phase, &abort_flag, g.status, 0x302);
        }
        if (!ok) {
            // copies under way land within microseconds; their barrier may be the other CTA's
            const unsigned long long t0 = tc::global_ns();
            while (tc::global_ns() - t0 < 5000000ull) {}
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = instr_desc_bf16(S::kTileM, BN, A_MN, B_MN);
            constexpr uint32_t kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;   // 16 of the reduction
            const uint32_t base = tc::smem_u32(tiles);
            int stage = 0, n = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = worker; t < total && ok; t += workers, ++n) {
                const Tile tile = decode(g, t);
                int k, k_end;
                k_range(g, tile, k, k_end);
                const int buf = n & 1;
                if (!(ok = warp_wait(&taken_bar[buf], ((n >> 1) & 1) ^ 1, &abort_flag, g.status, 0x303))) break;
                tc::tc_fence_after();
                const uint32_t acc = tmem + buf * BN;
                uint32_t accumulate = 0;
                for (; k < k_end; ++k) {
                    if (!(ok = warp_wait(&full_bar[stage], phase, &abort_flag, g.status, 0x304))) break;
                    tc::tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a = base + stage * S::kStageBytes;
                        const uint64_t da = smem_desc<A_MN>(a), db = smem_desc<B_MN>(a + S::kABytes);
                        mma_bf16<CG>(acc, da, db, idesc, accumulate);
#pragma unroll
                        for (int i = 1; i < kBlockK / 16; ++i) mma_bf16<CG>(acc, da + i * kStepA, db + i * kStepB, idesc, 1);
                        mma_commit<CG>(&empty_bar[stage]);
                    }
                    __syncwarp();
                    accumulate = 1;
                    if (++stage == S::kStages) { stage = 0; phase ^= 1; }
                }
                if (ok && elect_one()) mma_commit<CG>(&ready_bar[buf]);
                __syncwarp();
            }
            if (!ok) {
                if (elect_one()) mma_commit_here<CG>(&drain_bar);
                __syncwarp();
                const unsigned long long t0 = tc::global_ns();
                while (!tc::mbar_try_wait(&drain_bar, 0) && tc::global_ns() - t0 < tc::kWaitLimitNs) {}
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, part = (warp - 2) >> 2;
        constexpr int kPerWarp = kTileN * 4 / S::kEpilogueWarps;
        if (EPI == kEpiStore && g.bias.sums)
            fold_bias(g.bias, static_cast<long long>(blockIdx.x) * S::kEpilogueWarps + warp - 2, static_cast<long long>(gridDim.x) * S::kEpilogueWarps, lane);
        int n = 0;
        for (int t = worker; t < total; t += workers, ++n) {
            const Tile tile = decode(g, t);
            const Problem& p = g.p[tile.problem];
            const int buf = n & 1, N = p.N;
            const long long row = static_cast<long long>(tile.m) * S::kTileM + rank * kRows + quarter * 32 + lane;
            const int first = tile.n * kTileN + part * kPerWarp, columns = min(kPerWarp, N - first);   // may be none
            const bool in = row < p.M && g.splits == 1;       // the epilogue is applied here, or to the joined sum
            Fetched<EPI> fetched;                              // of the first columns: while the products still run
            if (in && columns > 0) epilogue_fetch<EPI>(p.e, row, first, N, fetched);
            // one lane asks for all
            bool ready = false;
            if (lane == 0) ready = tc::mbar_wait(&ready_bar[buf], (n >> 1) & 1, &abort_flag, g.status, 0x305);
            if (!__shfl_sync(0xFFFFFFFFu, ready, 0)) break;
            tc::tc_fence_after();
            const uint32_t acc = tmem + buf * BN + (static_cast<uint32_t>(quarter * 32) << 16) + part * kPerWarp;
            // Fetching the next columns' rows into a second set of registers gained nothing (the arithmetic then has fewer),
            // nor did asking the L2 for them a tile ahead (161 against 193 us for the block's first backward product).
            const auto release = [&] {                         // the accumulator has been read: the next products may have it
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 2) arrive_cluster(in_first_cta(&taken_bar[buf]));
                    else tc::mbar_arrive(&taken_bar[buf]);
                }
            };
#pragma unroll 1
            for (int c = 0; c < columns; c += kChunk) {
                const int col = first + c;
                if (in && c > 0) epilogue_fetch<EPI>(p.e, row, col, N, fetched);
                uint32_t raw[kChunk];
                Pair v[kChunk / 2], u[kChunk / 2];
                load_accumulator(acc + c, raw);
#pragma unroll
                for (int i = 0; i < kChunk / 2; ++i) v[i] = pair(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1]));
                if (EPI == kEpiGated) {
                    load_accumulator(acc + kTileN + c, raw);
#pragma unroll
                    for (int i = 0; i < kChunk / 2; ++i) u[i] = pair(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1]));
                }
                if (c + kChunk >= columns) release();
                if (in) {
                    epilogue_row<EPI>(p.e, row, col, N, fetched, v, u);
                } else if (row < p.M) {
                    const long long pitch = partial_pitch(N), plane = p.M * pitch;
                    float* to = g.partials + p.partial + tile.split * plane * (EPI == kEpiGated ? 2 : 1) + row * pitch + col;
                    store_row(to, kChunk, v);
                    if (EPI == kEpiGated) store_row(to + plane, kChunk, u);
                }
            }
            if (columns <= 0) release();
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

// Joins the partial sums of a split reduction in the pieces' order and applies the epilogue.  A CTA has 32 chunks of 32
// columns: its threads add four columns each, whole lines at a time and eight pieces under way, one warp does the epilogue.
template <int EPI>
__global__ void __launch_bounds__(256)
combine_kernel(const __grid_constant__ GemmArgs g) {
    constexpr int kParts = EPI == kEpiGated ? 2 : 1;
    __shared__ float4 sums[kParts][32][kChunk / 4 + 1];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const Problem& p = g.p[blockIdx.y];
    const long long pitch = partial_pitch(p.N), plane = p.M * pitch, step = plane * kParts, chunks = p.M * (pitch / kChunk);
    const long long first = static_cast<long long>(blockIdx.x) * 32;
    const float* from = g.partials + p.partial + (first * kChunk + 4 * threadIdx.x);
    if (first + threadIdx.x / 8 < chunks) {
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int s0 = 0; s0 < g.splits; s0 += 8) {
                float4 q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    q[j] = s0 + j < g.splits ? *reinterpret_cast<const float4*>(from + (s0 + j) * step + part * plane) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum.x += q[j].x; sum.y += q[j].y; sum.z += q[j].z; sum.w += q[j].w;
                }
            }
            sums[part][threadIdx.x / 8][threadIdx.x % 8] = sum;
        }
    }
    __syncthreads();
    const long long chunk = first + threadIdx.x;
    if (threadIdx.x >= 32 || chunk >= chunks) return;
    const long long row = chunk / (pitch / kChunk);
    const int col = static_cast<int>(chunk - row * (pitch / kChunk)) * kChunk;
    Fetched<EPI> f;
    epilogue_fetch<EPI>(p.e, row, col, p.N, f);
    Pair v[kChunk / 2], u[kChunk / 2];
#pragma unroll
    for (int j = 0; j < kChunk / 4; ++j) {
        const float4 q = sums[0][threadIdx.x][j];
        v[2 * j] = pair(q.x, q.y); v[2 * j + 1] = pair(q.z, q.w);
        if (EPI == kEpiGated) {
            const float4 w = sums[kParts - 1][threadIdx.x][j];
            u[2 * j] = pair(w.x, w.y); u[2 * j + 1] = pair(w.z, w.w);
        }
    }
    epilogue_row<EPI>(p.e, row, col, p.N, f, v, u);
}

}  // namespace lg
}  // namespace dynbatch
