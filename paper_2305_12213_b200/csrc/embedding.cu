// Embedding table: lookup with scaling, and the table's gradient by sorted tokens.
//     out[t] = scale * table[token[t]]          d_table[v] = scale * sum over t with token[t] = v of dy[t], t ascending
// Both are HBM-bound.  The gradient reads every row of dy once and writes every row of the table once: positions are
// sorted by token (stable, so that a row's sum has one order), the sorted list is cut into equal units whatever the
// tokens' frequencies are, a unit adds the rows of its runs of equal tokens in registers, and runs that reach over
// units are joined by a second small kernel from the units' partial sums.  No float atomics: the same call gives the
// same bits.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "common.h"
#include "layer_gemm.cuh"

namespace dynbatch {
namespace {

using bf16 = __nv_bfloat16;
using lg::Raw8;

constexpr int kBlock = 256;
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSortWarps = kBlock / 32, kSteps = 8;
constexpr int kPart = kBlock * kSteps;           // entries a CTA sorts at a time: 2048
constexpr int kMaxSortBlocks = 512;              // every CTA reads all CTAs' counts, so their number is bounded
constexpr int kClusterWarps = 32, kMaxSteps = 8, kMaxCluster = 8;   // sorting in one launch: up to 65536 rows
constexpr long long kClusterRows = 32LL * kClusterWarps * kMaxSteps * kMaxCluster;
constexpr int kFewRows = 256;                    // up to here nothing is sorted
constexpr long long kMaxRows = 1LL << 28, kMaxVocab = 1LL << 26, kMaxWidth = 1LL << 20;

long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------------------------- eight values of a row
__device__ __forceinline__ void store8(bf16* p, int n, const float (&v)[8]) {
    if (n == 8 && lg::aligned_to(p, 16)) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(lg::pack2(v[0], v[1]), lg::pack2(v[2], v[3]), lg::pack2(v[4], v[5]), lg::pack2(v[6], v[7])));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = __float2bfloat16_rn(v[j]);
    }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (n == 8 && lg::aligned_to(p, 16)) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = v[j];
    }
}

// ---------------------------------------------------------------------------------------------- lookup
struct LookupArgs {
    const int* tokens;
    const void* table;
    void* out;
    long long out_pitch, rows;
    int vocab, width;
    int threads_shift;
    float scale;
};

// threads_per_row threads (a power of two) take a row, 8 values each, blockIdx.y counts the parts of rows wider than that;
// a thread's four rows are all under way at once.  No division, no loop: CTAs come and go in the order of the rows.  HBM-bound
// (32768 tokens of 32000 x 2048 bf16, 8.8 thousand of them distinct: 29 to 32 us, where these rows of the table and the output,
// 171 MB, take 26 at the copy rate; some of the output is still in the L2 at the end).
constexpr int kLookupRows = 4;
template <class TT, class OT>
__global__ void __launch_bounds__(kBlock) embedding_kernel(const __grid_constant__ LookupArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int shift = a.threads_shift, groups = kBlock >> shift, group = threadIdx.x >> shift;
    const int col = ((blockIdx.y << shift) + (threadIdx.x & ((1 << shift) - 1))) * 8, n = min(8, a.width - col);
    if (n <= 0) return;
    const long long first = static_cast<long long>(blockIdx.x) * (kLookupRows * groups) + group;
    int token[kLookupRows];
    Raw8<TT> v[kLookupRows];
#pragma unroll
    for (int d = 0; d < kLookupRows; ++d) {
        const long long row = first + d * groups;
        token[d] = row < a.rows ? a.tokens[row] : -1;
    }
#pragma unroll
    for (int d = 0; d < kLookupRows; ++d) {
        const bool in = token[d] >= 0 && token[d] < a.vocab;
        v[d].load(static_cast<const TT*>(a.table) + static_cast<long long>(in ? token[d] : 0) * a.width + col, in ? n : 0);
    }
#pragma unroll
    for (int d = 0; d < kLookupRows; ++d) {
        const long long row = first + d * groups;
        if (row >= a.rows) break;
        float x[8];
        v[d].values(x);
        if (token[d] >= 0 && token[d] < a.vocab) {             // else zeros whatever the scale is
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= a.scale;
        }
        store8(static_cast<OT*>(a.out) + row * a.out_pitch + col, n, x);
    }
}

// ---------------------------------------------------------------------------------------------- rows without a token
// The rows of the table that no token names are zero.  Which they are takes no sort: each of these CTAs has every 2^shift-th
// row (so that all of them write into one moving window of the table), reads all tokens (from L2) and marks those of its
// share, then writes the rows that stayed unmarked.  The kernel is launched behind the sort, which occupies eight SMs, and
// runs beside it: the sort releases it only when all before the sort is complete, it touches nothing of the sort's, and it
// waits for the sort at its end, so that what follows it follows both.  (32768 tokens of 32000 x 2048 fp32: 90 us for the
// whole gradient, against 111 with these rows written by the kernel that adds; 23.3 thousand rows of 8 KB, 29 us at the copy
// rate, take 37.)
struct ZeroArgs {
    const int* tokens;
    unsigned char* out;
    long long row_bytes;
    int rows, vocab;
    int shift;                    // log2 of the number of CTAs
};
constexpr int kMarks = 8192;      // rows marked at a time

// `threads` threads (a power of two) write one row: 2-byte steps up to the first 16-byte boundary and behind the last
__device__ __forceinline__ void zero_row(unsigned char* p, long long bytes, int thread, int threads) {
    const long long lead = min(bytes, static_cast<long long>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15));
    const long long whole = (bytes - lead) / 16, tail = bytes - lead - 16 * whole;
    for (long long i = thread; i < whole; i += threads) __stcs(reinterpret_cast<uint4*>(p + lead) + i, make_uint4(0, 0, 0, 0));
    for (int i = thread; i < static_cast<int>(lead + tail) / 2; i += threads) {
        const long long at = 2 * i < lead ? 2 * i : bytes - tail + (2 * i - lead);
        *reinterpret_cast<unsigned short*>(p + at) = 0;
    }
}
constexpr int kZeroThreads = 512, kMaxZeroShift = 8;
__global__ void __launch_bounds__(kZeroThreads) embedding_zero_kernel(const __grid_constant__ ZeroArgs z) {
    __shared__ unsigned char marks[kMarks];
    tc::griddep_launch_dependents();
    const int index = blockIdx.x, mask = (1 << z.shift) - 1;
    const int share = (z.vocab - index + mask) >> z.shift;     // rows index, index + 2^shift, ...
    // up to a warp for a row, so that a row's test and its address are looked at once
    const bool wide = lg::aligned_to(z.out, 16) && z.row_bytes % 16 == 0;
    const int per_row = static_cast<int>(z.row_bytes / 16);
    int shift = 0;
    while (shift < 5 && (1 << shift) < per_row) ++shift;
    const int threads = 1 << shift, groups = blockDim.x >> shift, group = threadIdx.x >> shift, thread = threadIdx.x & (threads - 1);
    for (int lo = 0; lo < share; lo += kMarks) {
        const int n = min(kMarks, share - lo);
        for (int i = threadIdx.x; i < n; i += blockDim.x) marks[i] = 0;
        __syncthreads();
        constexpr int kAhead = 16;
        for (int i = threadIdx.x; i < z.rows; i += kAhead * kZeroThreads) {
            int token[kAhead];                                 // all read before the first mark, which could be any byte
#pragma unroll
            for (int d = 0; d < kAhead; ++d) token[d] = i + d * kZeroThreads < z.rows ? z.tokens[i + d * kZeroThreads] : -1;
#pragma unroll
            for (int d = 0; d < kAhead; ++d) {
                const unsigned r = static_cast<unsigned>((token[d] >> z.shift) - lo);      // a negative token's is large
                if ((token[d] & mask) == index && r < static_cast<unsigned>(n)) marks[r] = 1;
            }
        }
        __syncthreads();
        for (int r = group; r < n; r += groups) {
            if (marks[r]) continue;
            unsigned char* p = z.out + ((static_cast<long long>(lo + r) << z.shift) + index) * z.row_bytes;
            if (wide) {
#pragma unroll 8
                for (int i = thread; i < per_row; i += threads) __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(0, 0, 0, 0));
            } else {
                zero_row(p, z.row_bytes, thread, threads);
            }
        }
        __syncthreads();
    }
    tc::griddep_wait();
}

// ---------------------------------------------------------------------------------------------- sorting positions by token
struct SortArgs {
    const int* tokens;            // first pass; tokens outside the table sort behind it, as key `vocab`
    const int2* in;               // entries (key, position)
    int2* out;
    int* counts;                  // [CTA][bin]
    int* joins;                   // number of runs to join, zeroed by the first pass
    int rows, vocab, per_block, shift, first;
};

__device__ __forceinline__ int key_of(const int* tokens, int vocab, int i) {
    const int t = tokens[i];
    return t >= 0 && t < vocab ? t : vocab;
}
__device__ __forceinline__ int digit_of(int key, int shift) { return (key >> shift) & (kBins - 1); }

__global__ void __launch_bounds__(kBlock) sort_count_kernel(const __grid_constant__ SortArgs a) {
    __shared__ int bins[kBins];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    for (int b = threadIdx.x; b < kBins; b += kBlock) bins[b] = 0;
    if (a.first && blockIdx.x == 0 && threadIdx.x == 0) *a.joins = 0;
    __syncthreads();
    const int begin = blockIdx.x * a.per_block, end = min(a.rows, begin + a.per_block);
    for (int i = begin + threadIdx.x; i < end; i += kBlock)
        atomicAdd(&bins[digit_of(a.first ? key_of(a.tokens, a.vocab, i) : a.in[i].x, a.shift)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kBlock) a.counts[blockIdx.x * kBins + b] = bins[b];
}

// Exclusive sum over the bins, two per thread of the first eight warps; `total` holds kBins values and is replaced.
__device__ __forceinline__ void scan_bins(int* total, int* warp_sum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int x = 0, y = 0, s = 0;
    if (tid < kBins / 2) {
        x = total[2 * tid]; y = total[2 * tid + 1];
        s = x + y;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xFFFFFFFFu, s, d);
            if (lane >= d) s += o;
        }
        if (lane == 31) warp_sum[warp] = s;
    }
    __syncthreads();
    if (tid < kBins / 2) {
        int before = s - x - y;
#pragma unroll
        for (int w = 0; w < kBins / 64; ++w) before += w < warp ? warp_sum[w] : 0;
        total[2 * tid] = before;
        total[2 * tid + 1] = before + x;
    }
    __syncthreads();
}

// Ranks of 32 * STEPS * WARPS consecutive entries by digit, stable: a warp's entries are consecutive, and within a step
// equal digits are ranked by lane.  counters[WARPS][kBins] becomes the number of equal digits in earlier warps.
template <int WARPS, int STEPS>
__device__ __forceinline__ void rank_entries(const int (&key)[STEPS], int shift, int entries_left, unsigned short* counters,
                                             int (&rank)[STEPS]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned short* mine = counters + warp * kBins;
    for (int b = lane; b < kBins / 8; b += 32) reinterpret_cast<uint4*>(mine)[b] = make_uint4(0, 0, 0, 0);
    __syncwarp();
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (s * 32 >= entries_left) break;                     // the same for the whole warp
        const bool in = s * 32 + lane < entries_left;
        const unsigned live = __ballot_sync(0xFFFFFFFFu, in);
        const int d = digit_of(key[s], shift);
        unsigned same = live;                                  // lanes with this digit, a vote for each bit (the match
#pragma unroll                                                 // instruction takes four times as long)
        for (int b = 0; b < kDigitBits; ++b) {
            const unsigned set = __ballot_sync(0xFFFFFFFFu, (d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const int below = __popc(same & ((1u << lane) - 1));
        const int before = mine[d];
        rank[s] = before + below;
        __syncwarp();
        if (in && below == 0) mine[d] = static_cast<unsigned short>(before + __popc(same));
        __syncwarp();
    }
}

__global__ void __launch_bounds__(kBlock) sort_scatter_kernel(const __grid_constant__ SortArgs a) {
    __shared__ __align__(16) unsigned short counters[kSortWarps * kBins];
    __shared__ int base[kBins], total[kBins], warp_sum[kSortWarps];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int b = tid; b < kBins; b += kBlock) {
        int before = 0, all = 0;
#pragma unroll 8
        for (int j = 0; j < static_cast<int>(gridDim.x); ++j) {
            const int c = a.counts[j * kBins + b];
            all += c;
            if (j < static_cast<int>(blockIdx.x)) before += c;
        }
        base[b] = before;
        total[b] = all;
    }
    __syncthreads();
    scan_bins(total, warp_sum);
    for (int b = tid; b < kBins; b += kBlock) base[b] += total[b];
    __syncthreads();
    const int begin = blockIdx.x * a.per_block, end = min(a.rows, begin + a.per_block);
    for (int part = begin; part < end; part += kPart) {
        const int first = part + warp * 32 * kSteps;
        const int left = max(0, min(32 * kSteps, end - first));
        int key[kSteps], pos[kSteps], rank[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int i = first + s * 32 + lane;
            const bool in = s * 32 + lane < left;
            int2 x = make_int2(0, 0);
            if (in) x = a.first ? make_int2(key_of(a.tokens, a.vocab, i), i) : a.in[i];
            key[s] = x.x;
            pos[s] = x.y;
        }
        rank_entries<kSortWarps, kSteps>(key, a.shift, left, counters, rank);
        __syncthreads();
        for (int b = tid; b < kBins; b += kBlock) {       // counts become the start of each warp's entries
            unsigned short c[kSortWarps];
            int at = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) c[w] = counters[w * kBins + b];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                counters[w * kBins + b] = static_cast<unsigned short>(at);
                at += c[w];
            }
            total[b] = at;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s * 32 + lane < left) {
                const int d = digit_of(key[s], a.shift);
                const int to = base[d] + counters[warp * kBins + d] + rank[s];
                a.out[to] = make_int2(key[s], pos[s]);
            }
        }
        __syncthreads();
        for (int b = tid; b < kBins; b += kBlock) base[b] += total[b];
        __syncthreads();
    }
}

// All passes in one launch: up to eight CTAs of a cluster, each with a part of the entries in its registers.  A pass needs
// every CTA's counts for the place of a digit's entries, which they read from each other's shared memory; entries change
// hands through global memory, or shared memory where there is one CTA.  Bound by the scattered stores of the few CTAs:
// 300 tokens 8 us, 8192 12, 32768 18, 65536 38 (two passes).
struct ClusterSortArgs {
    const int* tokens;
    int2* between[2];             // entries (key, position) from pass to pass; the last pass writes [0]
    int* joins;
    int rows, vocab, passes, steps;   // a CTA has 1024 * steps entries
};
constexpr int kClusterThreads = 32 * kClusterWarps;
constexpr int kClusterSmem = 2 * kClusterThreads * kMaxSteps * 4 + kClusterWarps * kBins * 2;

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();                                  // .aligned: behind stores that only lanes with an entry made
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int load_cluster(const int* p, int rank) {
    int v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.s32 %0, [a];\n\t}"
                 : "=r"(v) : "r"(tc::smem_u32(p)), "r"(rank) : "memory");
    return v;
}

__global__ void __launch_bounds__(kClusterThreads) cluster_sort_kernel(const __grid_constant__ ClusterSortArgs a) {
    extern __shared__ int sort_smem[];
    int2* own = reinterpret_cast<int2*>(sort_smem);   // one CTA: the entries between passes
    unsigned short* counters = reinterpret_cast<unsigned short*>(sort_smem + 2 * kClusterThreads * kMaxSteps);
    __shared__ int counts[kBins], base[kBins], warp_sum[kClusterWarps];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, ctas = gridDim.x, rank = blockIdx.x;
    if (rank == 0 && tid == 0) *a.joins = 0;
    // consecutive entries for each warp
    const int first = (rank * kClusterWarps + warp) * 32 * a.steps, left = max(0, min(32 * a.steps, a.rows - first));
    int key[kMaxSteps], pos[kMaxSteps], where[kMaxSteps];
#pragma unroll
    for (int s = 0; s < kMaxSteps; ++s) {
        pos[s] = first + s * 32 + lane;
        key[s] = s * 32 + lane < left ? key_of(a.tokens, a.vocab, pos[s]) : 0;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * kDigitBits;
        rank_entries<kClusterWarps, kMaxSteps>(key, shift, left, counters, where);
        __syncthreads();
        if (tid < kBins) {
            unsigned short c[kClusterWarps];                   // read first: a chain of reads and writes costs 0.6 us
            int at = 0;
#pragma unroll
            for (int w = 0; w < kClusterWarps; ++w) c[w] = counters[w * kBins + tid];
#pragma unroll
            for (int w = 0; w < kClusterWarps; ++w) {
                counters[w * kBins + tid] = static_cast<unsigned short>(at);
                at += c[w];
            }
            counts[tid] = at;
        }
        if (ctas > 1) cluster_sync(); else __syncthreads();
        int before = 0;
        if (tid < kBins) {
            int all = 0, x[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) x[c] = c >= ctas ? 0 : ctas > 1 ? load_cluster(&counts[tid], c) : counts[tid];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) {
                all += x[c];
                if (c < rank) before += x[c];
            }
            base[tid] = all;
        }
        __syncthreads();
        scan_bins(base, warp_sum);
        if (tid < kBins) base[tid] += before;
        __syncthreads();
        const bool last = pass + 1 == a.passes;
        int2* to = last || ctas > 1 ? a.between[(a.passes - 1 - pass) & 1] : own;
#pragma unroll
        for (int s = 0; s < kMaxSteps; ++s) {
            if (s * 32 + lane < left) {
                const int d = digit_of(key[s], shift);
                const int at = base[d] + counters[warp * kBins + d] + where[s];
                to[at] = make_int2(key[s], pos[s]);
            }
        }
        if (last) break;
        if (ctas > 1) cluster_sync(); else __syncthreads();
#pragma unroll
        for (int s = 0; s < kMaxSteps; ++s) {
            if (s * 32 + lane < left) {
                const int2 x = to[first + s * 32 + lane];
                key[s] = x.x;
                pos[s] = x.y;
            }
        }
        __syncthreads();
    }
    if (ctas > 1) cluster_sync();                  // nobody leaves while others read its counts
}

// ---------------------------------------------------------------------------------------------- sums of runs
struct SumArgs {
    const int2* entries;          // (key, position), sorted
    const void* dy; long long dy_pitch;
    void* out;
    float* head; float* tail;     // [unit][width]: the part of a cut run that came from an earlier unit, that goes on in the next
    int* joins; int* join_list;   // units in which a cut run begins
    int rows, vocab, width;
    int unit, units;              // sorted entries per unit
    int threads_shift;            // log2 of the threads that take a row, 8 columns each
    float scale;
};

// A unit adds the runs of equal tokens that begin in it; one that reaches into the next unit it follows to its end.  Only
// runs that reach further, past the end of the next unit, are cut at the units' borders (few tokens are that frequent).
// HBM-bound: 31.8 thousand rows of 4 KB to 8.7 thousand of 8 KB, 201 MB, in 42 us, 0.73 of the copy rate.
template <class DT, class OT>
__global__ void __launch_bounds__(kBlock, sizeof(DT) == 2 ? 4 : 3) embedding_sum_kernel(const __grid_constant__ SumArgs a) {
    constexpr int kDeep = 4;                                    // rows under way
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int shift = a.threads_shift, group = threadIdx.x >> shift, groups = kBlock >> shift;
    const int col = ((blockIdx.y << shift) + (threadIdx.x & ((1 << shift) - 1))) * 8, n = min(8, a.width - col);
    if (n <= 0) return;
    OT* out = static_cast<OT*>(a.out);
    const int unit = blockIdx.x * groups + group;
    if (unit >= a.units) return;
    const int begin = unit * a.unit, end = min(a.rows, begin + a.unit);
    const DT* dy = static_cast<const DT*>(a.dy);
    const int head = a.entries[begin].x, last = a.entries[end - 1].x;
    const int beyond = end < a.rows ? a.entries[end].x : -1;
    // the run at the beginning: its own, another unit's (skipped), or cut
    const bool from_before = begin > 0 && a.entries[begin - 1].x == head;
    const bool head_cut = from_before && ((begin > a.unit && a.entries[begin - a.unit - 1].x == head) || beyond == head);
    const int skip = from_before && !head_cut ? head : -1;
    // the run at the end, if it begins here and goes on
    const bool goes_on = beyond == last && !(from_before && last == head);
    const bool tail_cut = goes_on && end + a.unit < a.rows && a.entries[end + a.unit].x == last;
    const int stop = goes_on && !tail_cut ? a.rows : end;
    int current = head;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    const auto flush = [&](bool cut) {
        if (current >= a.vocab || current == skip) return;
        if (head_cut && current == head) {
            store8(a.head + static_cast<long long>(unit) * a.width + col, n, sum);
        } else if (cut) {
            store8(a.tail + static_cast<long long>(unit) * a.width + col, n, sum);
            if (col == 0) a.join_list[atomicAdd(a.joins, 1)] = unit;
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = sum[j] * a.scale;
            store8(out + static_cast<long long>(current) * a.width + col, n, v);
        }
    };
    int key[kDeep], pos[kDeep];
    const auto entries = [&](int i) {                           // behind the unit's end only the last run counts
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const bool in = i + d < stop;
            const int2 x = in ? a.entries[i + d] : make_int2(-1, 0);
            key[d] = x.x;
            pos[d] = x.y;
        }
    };
    entries(begin);
    for (int i = begin; i < stop; i += kDeep) {
        Raw8<DT> v[kDeep];
        int now[kDeep];
        bool over = false;
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            now[d] = key[d];
            if (i + d >= end && now[d] != last) now[d] = -1;
            over = over || now[d] < 0;
            const bool in = now[d] >= 0 && now[d] < a.vocab && now[d] != skip;
            v[d].load(dy + static_cast<long long>(in ? pos[d] : 0) * a.dy_pitch + col, in ? n : 0);
        }
        if (!over) entries(i + kDeep);                          // the next entries, while the rows are under way
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            if (now[d] < 0) break;
            if (now[d] != current) {
                flush(false);
                current = now[d];
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = 0.f;
            }
            float x[8];
            v[d].values(x);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += x[j];
        }
        if (over) break;
    }
    flush(tail_cut);
}

// Few rows: no sort.  A warp holds all tokens, eight a lane, and asks for each of its rows of the table which of them are
// that row's token (at most eight votes); 256 columns a warp.  One launch, bound by its latency and the table's rows.
struct FewArgs {
    const int* tokens;
    const void* dy; long long dy_pitch;
    void* out;
    int rows, vocab, width;
    float scale;
};
template <class DT, class OT>
__global__ void __launch_bounds__(kBlock) embedding_few_kernel(const __grid_constant__ FewArgs a) {
    constexpr int kHeld = kFewRows / 32, kDeep = 4;
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = (blockIdx.y * 32 + lane) * 8, n = max(0, min(8, a.width - col));
    int token[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) token[j] = j * 32 + lane < a.rows ? a.tokens[j * 32 + lane] : -1;
    const int stride = gridDim.x * (kBlock / 32);
    for (int v = blockIdx.x * (kBlock / 32) + warp; v < a.vocab; v += stride) {
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
        bool named = false;                                     // a row that no token names is zeros whatever the scale is
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            unsigned found = __ballot_sync(0xFFFFFFFFu, token[h] == v);
            named = named || found;
            while (found) {                                     // the same for the whole warp; ascending rows
                Raw8<DT> x[kDeep];
                bool in[kDeep];
#pragma unroll
                for (int d = 0; d < kDeep; ++d) {
                    in[d] = found != 0;
                    const int row = in[d] ? h * 32 + __ffs(found) - 1 : 0;
                    found &= found - 1;
                    x[d].load(static_cast<const DT*>(a.dy) + row * a.dy_pitch + col, in[d] ? n : 0);
                }
#pragma unroll
                for (int d = 0; d < kDeep; ++d) {
                    if (!in[d]) break;
                    float y[8];
                    x[d].values(y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += y[j];
                }
            }
        }
        if (named) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
        }
        if (n > 0) store8(static_cast<OT*>(a.out) + static_cast<long long>(v) * a.width + col, n, sum);
    }
}

// Cut runs: the beginning's sum, then the units' in a fixed order (eight warps, each every eighth unit).
template <class OT>
__global__ void __launch_bounds__(kBlock) embedding_join_kernel(const __grid_constant__ SumArgs a) {
    constexpr int kWarps = kBlock / 32, kDeep = 4;
    __shared__ float part[kWarps][32 * 8 + 8];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slices = (a.width + 255) / 256, joins = *a.joins;
    for (long long i = blockIdx.x; i < static_cast<long long>(joins) * slices; i += gridDim.x) {
        const int unit = a.join_list[i / slices], col = static_cast<int>(i % slices) * 256 + lane * 8, n = max(0, min(8, a.width - col));
        const int key = a.entries[min(a.rows, (unit + 1) * a.unit) - 1].x;
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
        if (warp == 0) {
            Raw8<float> t;
            t.load(a.tail + static_cast<long long>(unit) * a.width + col, n);
            t.values(sum);
        }
        bool more = true;
        for (int u = unit + 1 + warp; more; u += kWarps * kDeep) {
            Raw8<float> v[kDeep];
            bool in[kDeep];
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                const int w = u + d * kWarps;
                in[d] = w < a.units && a.entries[static_cast<long long>(w) * a.unit].x == key;
                v[d].load(a.head + static_cast<long long>(w < a.units ? w : unit) * a.width + col, w < a.units ? n : 0);
            }
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                float x[8];
                v[d].values(x);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += in[d] ? x[j] : 0.f;
            }
            more = in[kDeep - 1];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) part[warp][lane * 8 + j] = sum[j];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int w = 1; w < kWarps; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += part[w][lane * 8 + j];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
            if (n > 0) store8(static_cast<OT*>(a.out) + static_cast<long long>(key) * a.width + col, n, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------- host
struct Launch {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    Launch(dim3 grid, int block, size_t smem, cudaStream_t stream, int cluster = 1) {
        std::memset(&cfg, 0, sizeof cfg);
        cfg.gridDim = grid;
        cfg.blockDim = dim3(block);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 2 : 1;
    }
    Launch(const Launch&) = delete;
    Launch& operator=(const Launch&) = delete;
};

bool valid_size(long long rows, long long vocab, long long width) {
    return rows >= 0 && rows <= kMaxRows && vocab >= 1 && vocab <= kMaxVocab && width >= 1 && width <= kMaxWidth &&
           rows * width <= (1LL << 40) && vocab * width <= (1LL << 40);
}

// Entries per unit: few enough that short batches fill the GPU, enough that partial sums stay rare in long ones.
int unit_of(long long rows) { return rows <= 4096 ? 8 : rows <= 16384 ? 16 : 32; }

struct GradLayout {
    size_t entries[2], counts, joins, join_list, head, tail, total;
    int unit, units;
};
GradLayout grad_layout(long long rows, long long width) {
    GradLayout L;
    size_t at = 0;
    const auto take = [&](long long bytes) {
        const size_t p = at;
        at += (static_cast<size_t>(bytes) + 255) / 256 * 256;
        return p;
    };
    L.unit = unit_of(rows);
    L.units = static_cast<int>(cdiv(rows, L.unit));
    for (int i = 0; i < 2; ++i) {
        L.entries[i] = take(8 * rows);
    }
    L.counts = take(4LL * kBins * std::min<long long>(kMaxSortBlocks, cdiv(rows, kPart)));
    L.joins = take(4);
    L.join_list = take(4LL * L.units);
    L.head = take(4LL * L.units * width);
    L.tail = take(4LL * L.units * width);
    L.total = at + 256;
    return L;
}

bool apart(const void* a, long long na, const void* b, long long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na <= 0 || nb <= 0 || x + static_cast<uintptr_t>(na) <= y || y + static_cast<uintptr_t>(nb) <= x;
}
int size_of(db_dtype t) { return t == DB_F32 ? 4 : 2; }
bool valid_type(db_dtype t) { return t == DB_F32 || t == DB_BF16; }

// Once per device: the attribute call costs a microsecond.
db_status allow_sort_smem() {
    constexpr int kDevices = 64;
    static std::atomic<unsigned char> done[kDevices];
    int device = 0;
    DB_CUDA_TRY(cudaGetDevice(&device));
    const bool known = device >= 0 && device < kDevices;
    if (known && done[device].load(std::memory_order_relaxed)) return DB_OK;
    DB_CUDA_TRY(cudaFuncSetAttribute(cluster_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kClusterSmem));
    if (known) done[device].store(1, std::memory_order_relaxed);
    return DB_OK;
}

// log2 of the threads that take a row, 8 values each
int shift_of(long long width) {
    int s = 0;
    while ((1 << s) < kBlock && (8LL << s) < width) ++s;
    return s;
}

template <class DT, class OT>
db_status launch_sum(const SumArgs& a, dim3 grid, cudaStream_t stream) {
    Launch S(grid, kBlock, 0, stream);
    DB_CUDA_TRY(cudaLaunchKernelEx(&S.cfg, embedding_sum_kernel<DT, OT>, a));
    if (a.units > 2) {                                          // a cut run is longer than a unit
        Launch J(dim3(static_cast<unsigned>(std::min<long long>(4LL * sm_count(), static_cast<long long>(a.units) * cdiv(a.width, 256)))), kBlock, 0, stream);
        DB_CUDA_TRY(cudaLaunchKernelEx(&J.cfg, embedding_join_kernel<OT>, a));
    }
    return DB_OK;
}

}  // namespace
}  // namespace dynbatch

extern "C" db_status db_embedding(const int32_t* tokens, const void* table, db_dtype table_dtype, float scale, int64_t rows,
                                  int32_t vocab, int32_t width, void* out, int64_t out_pitch, db_dtype out_dtype,
                                  void* cuda_stream) {
    using namespace dynbatch;
    if (!valid_size(rows, vocab, width)) return DB_ERR_ARG;
    if (!valid_type(table_dtype) || !valid_type(out_dtype)) return DB_ERR_UNSUPPORTED;
    if (!table || (rows > 0 && (!tokens || !out))) return DB_ERR_NULL;
    const int ts = size_of(table_dtype), os = size_of(out_dtype);
    if (rows > 0 && (out_pitch < width || out_pitch > (1LL << 31))) return DB_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(table) % ts || reinterpret_cast<uintptr_t>(out) % os) return DB_ERR_ARG;
    if (rows == 0) return DB_OK;
    const long long no = ((rows - 1) * out_pitch + width) * os;
    if (!apart(out, no, tokens, 4 * rows) || !apart(out, no, table, static_cast<long long>(vocab) * width * ts)) return DB_ERR_ARG;
    const int shift = shift_of(width);
    const LookupArgs a{tokens, table, out, out_pitch, rows, vocab, width, shift, scale};
    const long long per_cta = static_cast<long long>(kLookupRows) * (kBlock >> shift);
    Launch L(dim3(static_cast<unsigned>(cdiv(rows, per_cta)), static_cast<unsigned>(cdiv(width, 8LL << shift))), kBlock, 0,
             static_cast<cudaStream_t>(cuda_stream));
    void (*fn)(const LookupArgs) = table_dtype == DB_F32 ? (out_dtype == DB_F32 ? embedding_kernel<float, float> : embedding_kernel<float, bf16>)
                                                         : (out_dtype == DB_F32 ? embedding_kernel<bf16, float> : embedding_kernel<bf16, bf16>);
    DB_CUDA_TRY(cudaLaunchKernelEx(&L.cfg, fn, a));
    return DB_OK;
}

extern "C" size_t db_embedding_grad_workspace_bytes(int64_t rows, int32_t vocab, int32_t width) {
    using namespace dynbatch;
    return valid_size(rows, vocab, width) ? grad_layout(rows, width).total : 0;
}

extern "C" db_status db_embedding_grad(const int32_t* tokens, const void* dy, int64_t dy_pitch, db_dtype dy_dtype, float scale,
                                       int64_t rows, int32_t vocab, int32_t width, void* dtable, db_dtype grad_dtype,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
    using namespace dynbatch;
    if (!valid_size(rows, vocab, width)) return DB_ERR_ARG;
    if (!valid_type(dy_dtype) || !valid_type(grad_dtype)) return DB_ERR_UNSUPPORTED;
    if (!dtable || !workspace || (rows > 0 && (!tokens || !dy))) return DB_ERR_NULL;
    const int ds = size_of(dy_dtype), gs = size_of(grad_dtype);
    if (rows > 0 && (dy_pitch < width || dy_pitch > (1LL << 31))) return DB_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(dy) % ds || reinterpret_cast<uintptr_t>(dtable) % gs ||
        reinterpret_cast<uintptr_t>(workspace) % 256)
        return DB_ERR_ARG;
    const GradLayout L = grad_layout(rows, width);
    if (workspace_bytes < L.total) return DB_ERR_ARG;
    const long long nd = rows > 0 ? ((rows - 1) * dy_pitch + width) * ds : 0, ng = static_cast<long long>(vocab) * width * gs;
    const long long nw = static_cast<long long>(workspace_bytes);
    if (!apart(dtable, ng, dy, nd) || !apart(dtable, ng, tokens, 4 * rows) || !apart(dtable, ng, workspace, nw) ||
        !apart(workspace, nw, dy, nd) || !apart(workspace, nw, tokens, 4 * rows))
        return DB_ERR_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {
        DB_CUDA_TRY(cudaMemsetAsync(dtable, 0, static_cast<size_t>(ng), stream));
        return DB_OK;
    }
    if (rows <= kFewRows) {
        const FewArgs f{tokens, dy, dy_pitch, dtable, static_cast<int>(rows), vocab, width, scale};
        Launch F(dim3(static_cast<unsigned>(std::min<long long>(cdiv(vocab, kBlock / 32), 8LL * sm_count())), static_cast<unsigned>(cdiv(width, 256))),
                 kBlock, 0, stream);
        void (*fn)(const FewArgs) = dy_dtype == DB_F32 ? (grad_dtype == DB_F32 ? embedding_few_kernel<float, float> : embedding_few_kernel<float, bf16>)
                                                       : (grad_dtype == DB_F32 ? embedding_few_kernel<bf16, float> : embedding_few_kernel<bf16, bf16>);
        DB_CUDA_TRY(cudaLaunchKernelEx(&F.cfg, fn, f));
        return DB_OK;
    }
    char* base = static_cast<char*>(workspace);
    const auto ints = [&](size_t at) { return reinterpret_cast<int*>(base + at); };
    const auto entries = [&](int i) { return reinterpret_cast<int2*>(base + L.entries[i]); };
    // digits of 9 bits until the largest key, vocab (a token outside the table), is covered
    int passes = 1;
    while (vocab >> (passes * kDigitBits)) ++passes;
    int sorted = 0;
    ZeroArgs zero{tokens, static_cast<unsigned char*>(dtable), static_cast<long long>(width) * gs, static_cast<int>(rows), vocab, 0};
    // up to 256 CTAs, with eight rows at least
    while (zero.shift < kMaxZeroShift && (16LL << zero.shift) <= vocab) ++zero.shift;
    if (rows <= kClusterRows) {
        // a CTA for each 1024 rows, up to eight, then more entries for each
        int ctas = 1;
        while (ctas < kMaxCluster && ctas * kClusterThreads < rows) ctas *= 2;
        ClusterSortArgs s{};
        s.tokens = tokens;
        s.between[0] = entries(0);
        s.between[1] = entries(1);
        s.joins = ints(L.joins);
        s.rows = static_cast<int>(rows); s.vocab = vocab; s.passes = passes;
        s.steps = static_cast<int>(cdiv(rows, static_cast<long long>(ctas) * kClusterThreads));
        const db_status st = allow_sort_smem();
        if (st != DB_OK) return st;
        Launch S(dim3(ctas), kClusterThreads, kClusterSmem, stream, ctas), Z(dim3(1 << zero.shift), kZeroThreads, 0, stream);
        DB_CUDA_TRY(cudaLaunchKernelEx(&S.cfg, cluster_sort_kernel, s));
        DB_CUDA_TRY(cudaLaunchKernelEx(&Z.cfg, embedding_zero_kernel, zero));
    } else {
        SortArgs s{};
        s.tokens = tokens; s.rows = static_cast<int>(rows); s.vocab = vocab;
        s.counts = ints(L.counts);
        s.joins = ints(L.joins);
        const int blocks = static_cast<int>(std::min<long long>(kMaxSortBlocks, cdiv(rows, kPart)));
        s.per_block = static_cast<int>(cdiv(cdiv(rows, blocks), kPart) * kPart);
        const int used = static_cast<int>(cdiv(rows, s.per_block));
        for (int p = 0; p < passes; ++p) {
            s.first = p == 0; s.shift = p * kDigitBits;
            s.in = entries((p + 1) & 1);
            s.out = entries(p & 1);
            sorted = p & 1;
            Launch C(dim3(used), kBlock, 0, stream), S(dim3(used), kBlock, 0, stream), Z(dim3(1 << zero.shift), kZeroThreads, 0, stream);
            DB_CUDA_TRY(cudaLaunchKernelEx(&C.cfg, sort_count_kernel, s));
            if (p == 0) DB_CUDA_TRY(cudaLaunchKernelEx(&Z.cfg, embedding_zero_kernel, zero));
            DB_CUDA_TRY(cudaLaunchKernelEx(&S.cfg, sort_scatter_kernel, s));
        }
    }
    SumArgs a{};
    a.entries = entries(sorted);
    a.dy = dy; a.dy_pitch = dy_pitch; a.out = dtable;
    a.head = reinterpret_cast<float*>(base + L.head); a.tail = reinterpret_cast<float*>(base + L.tail);
    a.joins = ints(L.joins); a.join_list = ints(L.join_list);
    a.rows = static_cast<int>(rows); a.vocab = vocab; a.width = width;
    a.unit = L.unit; a.units = L.units; a.scale = scale;
    a.threads_shift = shift_of(width);
    const int groups = kBlock >> a.threads_shift;
    const dim3 grid(static_cast<unsigned>(cdiv(L.units, groups)), static_cast<unsigned>(cdiv(width, 8LL << a.threads_shift)));
    if (dy_dtype == DB_F32) return grad_dtype == DB_F32 ? launch_sum<float, float>(a, grid, stream) : launch_sum<float, bf16>(a, grid, stream);
    return grad_dtype == DB_F32 ? launch_sum<bf16, float>(a, grid, stream) : launch_sum<bf16, bf16>(a, grid, stream);
}
