// The layers whose gradients the workers send: linear layer and gated feed-forward block, forward and backward
// (entry points, planning, and the small kernels around the products of layer_gemm.cuh).
#include <algorithm>
#include <atomic>
#include <cstring>

#include "common.h"
#include "dynbatch_bench.h"
#include "layer_gemm.cuh"
#include "tensor_map.h"

namespace dynbatch {
namespace {

using bf16 = __nv_bfloat16;
using lg::Pair;

constexpr size_t kStatusBytes = 256;
constexpr long long kMaxRows = 1LL << 30, kMaxFeatures = 1LL << 24, kMaxElements = 1LL << 40, kMaxPitch = 1LL << 31;

size_t round256(size_t x) { return (x + 255) / 256 * 256; }
__host__ __device__ constexpr long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------------------------- small kernels
// Copies of bf16 matrices to rows of `to_pitch` (a multiple of 8): what brings operands to the 16-byte grid that TMA needs (two
// operands of 333 x 1001 and 1001 x 777 4.5 us, most of it the launch).
struct Repitch {
    const bf16* from; bf16* to;
    long long from_pitch, to_pitch, rows;
    int cols;
};
constexpr int kMaxCopies = 5;
struct RepitchArgs {
    Repitch m[kMaxCopies];       // blockIdx.y
    int* clear_status;
};
__global__ void __launch_bounds__(256) repitch_kernel(const __grid_constant__ RepitchArgs a) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    if (a.clear_status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.clear_status = 0;
    const Repitch& m = a.m[blockIdx.y];
    const long long per_row = cdiv(m.cols, 8), total = m.rows * per_row;
    for (long long i = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < total; i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const long long r = i / per_row;
        const int c = static_cast<int>(i - r * per_row) * 8;
        lg::Raw8<bf16> x;
        x.load(m.from + r * m.from_pitch + c, min(8, m.cols - c));
        *reinterpret_cast<uint4*>(m.to + r * m.to_pitch + c) = x.q;
    }
}

struct ActGradArgs {
    const bf16* dy; long long dy_pitch;
    lg::Kept z;
    int z_e4m3, act;
    bf16* dz; long long dz_pitch;        // nullptr: not written
    float* sums; long long sums_pitch;   // [row slabs][sums_pitch] sums over the slab's rows, or nullptr
    long long rows;
    int cols, slab_rows;
    int* clear_status;
};

// dz = dy act'(z) and the sums of its columns.  HBM-bound (sums alone of 16384 x 2048: 13.6 us, 4.9 TB/s).  A warp takes 256 columns of a row, eight per lane; a CTA's
// eight warps take every eighth row of a slab and add their sums in warp order, so the result does not depend on timing.
template <int ACT, bool E4M3>
__global__ void __launch_bounds__(256)
act_grad_kernel(const __grid_constant__ ActGradArgs a) {
    __shared__ float part[8][256];
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    if (a.clear_status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.clear_status = 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = (blockIdx.x * 32 + lane) * 8, n = min(8, a.cols - col);
    const long long first = static_cast<long long>(blockIdx.y) * a.slab_rows, last = min(a.rows, first + a.slab_rows);
    Pair sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = lg::both(0.f);
    if (n > 0) {
        constexpr int kDeep = 4;                               // rows under way
        for (long long r0 = first + warp; r0 < last; r0 += 8 * kDeep) {
            lg::Raw8<bf16> dy[kDeep], z16[kDeep];
            lg::Codes8 z8[kDeep];
            uint32_t byte[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const long long r = r0 + 8 * i;
                const int m = r < last ? n : 0;
                dy[i].load(a.dy + r * a.dy_pitch + col, m);
                if (ACT == DB_ACT_NONE) continue;
                if (E4M3) {
                    byte[i] = m ? a.z.scale[r * ((a.cols + 31) / 32) + col / 32] : 0;
                    z8[i].load(static_cast<const uint8_t*>(a.z.data) + r * a.cols + col, m);
                } else {
                    z16[i].load(static_cast<const bf16*>(a.z.data) + r * a.cols + col, m);
                }
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const long long r = r0 + 8 * i;
                if (r >= last) break;
                Pair d[4];
                dy[i].values(d);
                if (ACT != DB_ACT_NONE) {
                    Pair z[4];
                    if (E4M3) z8[i].values(byte[i], z);
                    else z16[i].values(z);
                    lg::Batch value, slope;
                    lg::act_batch_slope<ACT>(z, value, slope);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = lg::mul(d[j], slope[j]);
                }
                if (a.dz) {
                    bf16* q = a.dz + r * a.dz_pitch + col;     // workspace rows: aligned, pitch a multiple of 32
                    if (n == 8) {
                        *reinterpret_cast<uint4*>(q) = make_uint4(lg::pack_pair(d[0]), lg::pack_pair(d[1]), lg::pack_pair(d[2]), lg::pack_pair(d[3]));
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float x, y;
                            lg::halves(d[j], x, y);
                            if (2 * j < n) q[2 * j] = __float2bfloat16_rn(x);
                            if (2 * j + 1 < n) q[2 * j + 1] = __float2bfloat16_rn(y);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = lg::add(sum[j], d[j]);
            }
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) lg::halves(sum[j], part[warp][lane * 8 + 2 * j], part[warp][lane * 8 + 2 * j + 1]);
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w][threadIdx.x];
        a.sums[blockIdx.y * a.sums_pitch + c] = s;
    }
}

using ActGradFn = void (*)(const ActGradArgs);
ActGradFn act_grad_fn(int act, bool e4m3) {
    switch (act) {
        case DB_ACT_RELU: return e4m3 ? act_grad_kernel<DB_ACT_RELU, true> : act_grad_kernel<DB_ACT_RELU, false>;
        case DB_ACT_GELU: return e4m3 ? act_grad_kernel<DB_ACT_GELU, true> : act_grad_kernel<DB_ACT_GELU, false>;
        case DB_ACT_SILU: return e4m3 ? act_grad_kernel<DB_ACT_SILU, true> : act_grad_kernel<DB_ACT_SILU, false>;
        default: return act_grad_kernel<DB_ACT_NONE, false>;
    }
}

// The column sums where no product follows that would finish them on the side.
__global__ void __launch_bounds__(128) bias_fold_kernel(const __grid_constant__ lg::BiasFold f) {
    tc::griddep_wait();
    tc::griddep_launch_dependents();
    lg::fold_bias(f, (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / 32, gridDim.x * (blockDim.x / 32), threadIdx.x & 31);
}

// ---------------------------------------------------------------------------------------------- launches
// Every kernel of a call may be scheduled while its predecessor still runs and waits for it on the device.
struct Launch {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    Launch(dim3 grid, dim3 block, size_t smem, cudaStream_t stream, int cluster = 1) {
        std::memset(&cfg, 0, sizeof cfg);
        cfg.gridDim = grid;
        cfg.blockDim = block;
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

struct Matrix {              // bf16, row-major
    const bf16* p = nullptr;
    long long rows = 0, cols = 0, pitch = 0;
};

bool on_grid(const void* p, long long pitch) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch % 8 == 0; }

// Boxes of box_rows rows x 64 columns with the 128-byte swizzle; what lies outside the matrix reads as zero.
db_status make_map(CUtensorMap* map, const Matrix& m, int box_rows) {
    const TensorMapSpec spec{CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p,
                             {static_cast<cuuint64_t>(m.cols), static_cast<cuuint64_t>(m.rows)},
                             {static_cast<cuuint64_t>(m.pitch) * 2},
                             {lg::kBlockK, static_cast<cuuint32_t>(box_rows)},
                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B};
    return encode_tensor_map(map, spec, "cuTensorMapEncodeTiled rejected an operand of a layer");
}

// ---------------------------------------------------------------------------------------------- the products' plan
enum Kind { kForward, kGated, kInputGrad, kGatedGrad, kWeightGrad };   // which operands lie how, and the epilogue
enum TileShape { kPair256, kPair128, kSingle128, kSingle64, kTileShapes };

using GemmFn = void (*)(const lg::GemmArgs);
struct ShapeInfo { int cg, bn, smem, ctas, threads; };
template <int CG, int BN> constexpr ShapeInfo info() {
    using S = lg::Shape<CG, BN>;
    return {CG, BN, S::kSmemBytes, S::kCtas, S::kThreads};
}
constexpr ShapeInfo kShapes[kTileShapes] = {info<2, 256>(), info<2, 128>(), info<1, 128>(), info<1, 64>()};

template <int CG, int BN>
GemmFn gemm_fn(Kind kind) {
    switch (kind) {
        case kForward: return lg::layer_gemm_kernel<CG, BN, false, true, lg::kEpiStore>;
        case kInputGrad: return lg::layer_gemm_kernel<CG, BN, false, false, lg::kEpiStore>;
        case kGatedGrad: return lg::layer_gemm_kernel<CG, BN, false, false, lg::kEpiGatedGrad>;
        case kWeightGrad: return lg::layer_gemm_kernel<CG, BN, true, true, lg::kEpiStore>;
        case kGated:
            if constexpr (BN >= 128) return lg::layer_gemm_kernel<CG, BN, false, true, lg::kEpiGated>;
            else return nullptr;
    }
    return nullptr;
}
GemmFn gemm_fn(Kind kind, TileShape shape) {
    switch (shape) {
        case kPair256: return gemm_fn<2, 256>(kind);
        case kPair128: return gemm_fn<2, 128>(kind);
        case kSingle128: return gemm_fn<1, 128>(kind);
        default: return gemm_fn<1, 64>(kind);
    }
}

struct Size { long long M, N; };
struct Plan {
    TileShape shape = kPair256;
    int splits = 1, blocks_per_split = 1;
    long long partial_floats = 0;
};

long long tiles_of(Kind kind, TileShape shape, const Size& s) {
    const int tile_n = kind == kGated ? kShapes[shape].bn / 2 : kShapes[shape].bn;
    return cdiv(s.M, lg::kRows * kShapes[shape].cg) * cdiv(s.N, tile_n);
}

// The tile shape and the number of pieces of the reduction with the least estimated time, in SM cycles.
// A 64-deep block of a tile costs its products or its copies (about 57 bytes a cycle reach an SM), whichever is longer,
// more for each of two CTAs on an SM; a tile something for its start and end; and a reduction in pieces a second kernel,
// which reads eight pieces at a time, and the traffic of the partial sums.  In 64-column tiles, us by pieces 1, 4, 8, 16:
// 256 x 2048 x 1000 11.9, 10.2, 9.3, 11.9; 16 x 2048 x 512 above 7.4, 7.3, 6.7, 6.8 (32: 8.4); 1000 x 1024 x 256 7.7, 8.7, 8.8;
// 1024 x 1024 x 1024 8.3, in two 14.4.  Replayed from a graph, us in pairs of 256 and 128 columns and single CTAs of 128 and 64
// (rows x n_in x n_out, each in its best number of pieces, the picked one in brackets):
//   y   256 x 2048 x 1000 11.8, 9.5, 11.6, [9.2]     1024 x 1024 x 1024 10.5, 8.8, 9.1, [8.4]     2048 x 1024 x 1024 10.9, [9.6], 9.7, 9.1
//       150 x 5536 x 1704 13.4, [12.6], 16.0, 15.2   4100 x 320 x 640 7.5, 7.5, [6.8], 7.0        3000 x 1032 x 1544 [21.1], 22.2, 30.8, 32.9
//       2000 x 4096 x 1024 25.3, [22.2], 24.3, 23.1  8191 x 1024 x 4096 [48.4], 69.0, 64.1, 84.2
//   dx  9236 x 136 x 1088 11.4, [9.8], 10.1, 10.3    2050 x 1096 x 2184 [20.4], 23.7, 31.5, 35.9  8191 x 1024 x 4096 [50.3], 71.5, 61.8, 82.1
//   dW  129 x 1568 x 4608 9.5, 10.6, [9.1], 10.1     3000 x 1032 x 1544 24.6, [20.7], 24.4, 31.8  8191 x 1024 x 4096 [49.9], 72.4, 62.6, 83.8
// Of 39 products looked at this way the pick was within 7 % of the best but for one: dW of 5000 x 520 x 1032 took 22.2 in single
// CTAs of 128 columns and six pieces, 19.7 in pairs of 256 and four.  What follows the product is not in the estimate.
Plan make_plan(Kind kind, const Size* sizes, int n, long long blocks) {
    constexpr double kBlock[kTileShapes] = {560, 430, 560, 380}, kShared[kTileShapes] = {560, 430, 900, 550};
    constexpr double kTile[kTileShapes] = {4700, 3100, 1500, 1300}, kCombine = 4500, kEight = 1000;
    Plan best;
    if (blocks == 0 || n == 0) return best;                  // no rows: nothing is launched
    for (int j = 0; j < n; ++j)
        if (sizes[j].M == 0) return best;
    const int sms = sm_count();
    double least = 0;
    for (int i = 0; i < kTileShapes; ++i) {
        const TileShape shape = static_cast<TileShape>(i);
        if (!gemm_fn(kind, shape)) continue;
        const long long alone = std::max(1, sms / kShapes[i].cg), workers = alone * kShapes[i].ctas;
        long long tiles = 0, outputs = 0;
        for (int j = 0; j < n; ++j) {
            tiles += tiles_of(kind, shape, sizes[j]);
            outputs += sizes[j].M * lg::partial_pitch(sizes[j].N) * (kind == kGated ? 2 : 1);
        }
        for (long long want = std::min(blocks, std::max(1LL, workers / tiles));; want = (want + 1) / 2) {
            const long long per = cdiv(blocks, want), splits = cdiv(blocks, per), ctas = tiles * splits;
            const double time = static_cast<double>(cdiv(ctas, workers)) * per * (ctas > alone ? kShared[i] : kBlock[i]) + kTile[i] +
                                (splits > 1 ? kCombine + kEight * cdiv(splits, 8) + outputs * (splits + 1) * 4 / 6000.0 : 0);
            if (least == 0 || time < least) {
                least = time;
                best.shape = shape;
                best.splits = static_cast<int>(splits);
                best.blocks_per_split = static_cast<int>(per);
                best.partial_floats = splits > 1 ? splits * outputs : 0;
            }
            if (want == 1) break;
        }
    }
    return best;
}

// The products of the layers.  A call's workspace, its launches and db_bench_layer_plan take a product's plan from here.
Plan plan_forward(long long rows, long long n_in, long long n_out) {                // x w; h w_down
    const Size size{rows, n_out};
    return make_plan(kForward, &size, 1, cdiv(n_in, lg::kBlockK));
}
Plan plan_input_grad(long long rows, long long n_in, long long n_out, int sources) {   // dz w^T, or the sum of two of them
    const Size size{rows, n_in};
    return make_plan(kInputGrad, &size, 1, sources * cdiv(n_out, lg::kBlockK));
}
Plan plan_gated(long long rows, long long width, long long hidden) {                // gate and up
    const Size size{rows, hidden};
    return make_plan(kGated, &size, 1, cdiv(width, lg::kBlockK));
}
Plan plan_gated_grad(long long rows, long long width, long long hidden) {           // dh
    const Size size{rows, hidden};
    return make_plan(kGatedGrad, &size, 1, cdiv(width, lg::kBlockK));
}
Plan plan_weight_grad(const Size* sizes, int n, long long rows) {                   // x^T dz, up to three at once
    return make_plan(kWeightGrad, sizes, n, cdiv(rows, lg::kBlockK));
}

// Once per kernel and device: the attribute call costs a microsecond.
db_status allow_smem(Kind kind, TileShape shape, GemmFn fn, int bytes) {
    constexpr int kDevices = 64;
    static std::atomic<unsigned char> done[kDevices][kWeightGrad + 1][kTileShapes];
    int device = 0;
    DB_CUDA_TRY(cudaGetDevice(&device));
    const bool known = device >= 0 && device < kDevices;
    if (known && done[device][kind][shape].load(std::memory_order_relaxed)) return DB_OK;
    DB_CUDA_TRY(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (known) done[device][kind][shape].store(1, std::memory_order_relaxed);
    return DB_OK;
}

// One product, or several with the same reduction, in one launch (two with a split reduction).
struct Product {
    Matrix a[2], b[2];           // sources of the reduction; kGated: b[0], b[1] the two weights
    int sources = 1;
    Size size;
    lg::EpilogueArgs e;
};

long long depth(Kind kind, const Matrix& a) { return kind == kWeightGrad ? a.rows : a.cols; }

db_status run_products(Kind kind, const Plan& plan, const Product* products, int n, float* partials, int* status, bool& clear,
                       cudaStream_t stream, const lg::BiasFold& bias = {}) {
    const bool a_mn = kind == kWeightGrad, b_mn = kind != kInputGrad && kind != kGatedGrad;
    lg::GemmArgs g;
    std::memset(static_cast<void*>(&g), 0, sizeof g);
    for (int i = 0; i < n; ++i) {
        lg::Problem& p = g.p[i];
        p.M = static_cast<int>(products[i].size.M);
        p.N = static_cast<int>(products[i].size.N);
        p.blocks0 = static_cast<int>(cdiv(depth(kind, products[i].a[0]), lg::kBlockK));
        p.blocks = p.blocks0 + (products[i].sources > 1 ? static_cast<int>(cdiv(depth(kind, products[i].a[1]), lg::kBlockK)) : 0);
        p.e = products[i].e;
    }
    const ShapeInfo& shape = kShapes[plan.shape];
    const int tile_n = kind == kGated ? shape.bn / 2 : shape.bn;
    long long tiles = 0, floats = 0;
    for (int i = 0; i < n; ++i) {
        lg::Problem& p = g.p[i];
        p.m_tiles = static_cast<int>(cdiv(p.M, lg::kRows * shape.cg));
        p.n_tiles = static_cast<int>(cdiv(p.N, tile_n));
        p.partial = floats;
        floats += plan.splits * static_cast<long long>(p.M) * lg::partial_pitch(p.N) * (kind == kGated ? 2 : 1);
        g.tile_start[i] = static_cast<int>(tiles);
        tiles += static_cast<long long>(p.m_tiles) * p.n_tiles * plan.splits;
        const int sources = kind == kGated ? 2 : products[i].sources;
        db_status st;
        for (int s = 0; s < sources; ++s) {
            if (s < products[i].sources && (st = make_map(&p.a[s], products[i].a[s], a_mn ? lg::kBlockK : lg::kRows)) != DB_OK) return st;
            if ((st = make_map(&p.b[s], products[i].b[s], b_mn ? lg::kBlockK : shape.bn / shape.cg)) != DB_OK) return st;
        }
    }
    g.tile_start[n] = static_cast<int>(tiles);
    g.problems = n;
    g.splits = plan.splits;
    g.blocks_per_split = plan.blocks_per_split;
    g.partials = partials;
    g.status = status;
    g.clear_status = clear;
    g.bias = bias;
    clear = false;
    const GemmFn fn = gemm_fn(kind, plan.shape);
    const db_status st = allow_smem(kind, plan.shape, fn, shape.smem);
    if (st != DB_OK) return st;
    // as many CTAs (pairs) as fit share the tiles out
    const long long workers = std::min<long long>(std::max(1, sm_count() * shape.ctas / shape.cg), tiles);
    Launch L(dim3(static_cast<unsigned>(workers * shape.cg)), dim3(shape.threads), shape.smem, stream, shape.cg);
    DB_CUDA_TRY(cudaLaunchKernelEx(&L.cfg, fn, g));
    if (plan.splits > 1) {
        long long most = 0;
        for (int i = 0; i < n; ++i) most = std::max(most, static_cast<long long>(g.p[i].M) * (lg::partial_pitch(g.p[i].N) / lg::kChunk));
        Launch C(dim3(static_cast<unsigned>(cdiv(most, 32)), n), dim3(256), 0, stream);
        GemmFn fold = kind == kGated ? lg::combine_kernel<lg::kEpiGated> : kind == kGatedGrad ? lg::combine_kernel<lg::kEpiGatedGrad>
                                                                                            : lg::combine_kernel<lg::kEpiStore>;
        DB_CUDA_TRY(cudaLaunchKernelEx(&C.cfg, fold, g));
    }
    return DB_OK;
}

// ---------------------------------------------------------------------------------------------- workspace, arguments
struct Arena {               // hands out the workspace in pieces of whole 256 bytes; base may be null to count only
    char* base;
    size_t used = kStatusBytes;
    explicit Arena(void* p) : base(static_cast<char*>(p)) {}
    char* take(size_t bytes) {
        char* p = base ? base + used : nullptr;
        used += round256(bytes);
        return p;
    }
};

// An operand for TMA: the matrix itself where it lies on the 16-byte grid, else a copy in the workspace, made by copy_now().
struct Operands {
    Arena& arena;
    RepitchArgs copies{};
    int count = 0;
    long long most = 0;
    explicit Operands(Arena& a) : arena(a) {}
    Matrix of(const void* p, long long rows, long long cols, long long pitch) {
        Matrix m{static_cast<const bf16*>(p), rows, cols, pitch};
        if (on_grid(p, pitch)) return m;
        m.pitch = (cols + 7) / 8 * 8;
        bf16* to = reinterpret_cast<bf16*>(arena.take(static_cast<size_t>(rows * m.pitch) * 2));
        copies.m[count++] = {m.p, to, pitch, m.pitch, rows, static_cast<int>(cols)};
        most = std::max(most, rows * (m.pitch / 8));
        m.p = to;
        return m;
    }
    db_status copy_now(int* status, bool& clear, cudaStream_t stream) {
        if (count == 0) return DB_OK;
        copies.clear_status = clear ? status : nullptr;
        clear = false;
        Launch L(dim3(static_cast<unsigned>(std::min<long long>(cdiv(most, 256), 8LL * sm_count())), count), dim3(256), 0, stream);
        DB_CUDA_TRY(cudaLaunchKernelEx(&L.cfg, repitch_kernel, copies));
        return DB_OK;
    }
};

// Rows of `row` bytes, `pitch` bytes apart.
struct Extent {
    const void* p;
    long long rows, row, pitch;
    bool written;
};
Extent matrix(const void* p, long long rows, long long cols, long long pitch, int size, bool written) { return {p, rows, cols * size, pitch * size, written}; }
Extent block(const void* p, long long bytes, bool written) { return {p, bytes > 0 ? 1 : 0, bytes, bytes, written}; }

bool overlap(const Extent& x, const Extent& y) {
    if (!x.p || !y.p || x.rows < 1 || y.rows < 1) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    if (a >= b + static_cast<uintptr_t>((y.rows - 1) * y.pitch + y.row) || b >= a + static_cast<uintptr_t>((x.rows - 1) * x.pitch + x.row)) return false;
    if (x.pitch == y.pitch && x.rows > 1 && y.rows > 1) {      // columns of one tensor: apart if they are in every row
        const long long ahead = b >= a ? static_cast<long long>((b - a) % static_cast<uintptr_t>(x.pitch))
                                       : (x.pitch - static_cast<long long>((a - b) % static_cast<uintptr_t>(x.pitch))) % x.pitch;
        return ahead < x.row || ahead + y.row > x.pitch;
    }
    return true;
}
// Whether something that a call writes overlaps anything else it touches.
template <int N>
bool overlaps(const Extent (&x)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = i + 1; j < N; ++j)
            if ((x[i].written || x[j].written) && overlap(x[i], x[j])) return true;
    return false;
}

bool valid_size(long long rows, long long n_in, long long n_out) {
    return rows >= 0 && rows <= kMaxRows && n_in >= 1 && n_in <= kMaxFeatures && n_out >= 1 && n_out <= kMaxFeatures &&
           rows * n_in <= kMaxElements && rows * n_out <= kMaxElements && n_in * n_out <= kMaxElements;
}
bool valid_pitch(const void* p, long long cols, long long pitch) { return !p || (pitch >= cols && pitch <= kMaxPitch); }
bool odd_address(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }
bool valid_act(int act) { return act >= DB_ACT_NONE && act <= DB_ACT_SILU; }
long long scales_of(long long n) { return (n + ck8::kGroup - 1) / ck8::kGroup; }
int kept_size(db_dtype t) { return t == DB_E4M3 ? 1 : 2; }

db_status zero(void* p, long long bytes, cudaStream_t stream) {
    if (p && bytes > 0) DB_CUDA_TRY(cudaMemsetAsync(p, 0, static_cast<size_t>(bytes), stream));
    return DB_OK;
}

// ---------------------------------------------------------------------------------------------- linear layer
struct LinearArgs {
    const void *x, *w, *bias, *residual;
    long long x_pitch, residual_pitch, rows;
    int n_in, n_out, act;
    void* y;
    long long y_pitch;
    void *z, *z_scale;
    db_dtype z_dtype;
};

// Lays out the workspace and, with a base, launches; without one it only counts.
db_status linear_forward(const LinearArgs& v, Arena& arena, cudaStream_t stream, bool aligned) {
    int* status = reinterpret_cast<int*>(arena.base);
    bool clear = true;
    Operands ops(arena);
    Product p;
    const void* off = aligned ? nullptr : reinterpret_cast<const void*>(2);   // when counting: a pointer off the grid
    const bool count = !arena.base;
    const long long px = count ? (aligned ? (v.n_in + 7) / 8 * 8 : v.n_in) : v.x_pitch;
    p.a[0] = ops.of(count ? off : v.x, v.rows, v.n_in, px);
    p.b[0] = ops.of(count ? off : v.w, v.n_in, v.n_out, v.n_out);
    p.size = {v.rows, v.n_out};
    p.e.out = v.y; p.e.out_pitch = v.y_pitch;
    p.e.bias = static_cast<const bf16*>(v.bias);
    p.e.addend = static_cast<const bf16*>(v.residual); p.e.addend_pitch = v.residual_pitch;
    p.e.kept[0] = {v.z, static_cast<uint8_t*>(v.z_scale)};
    p.e.kept_e4m3 = v.z_dtype == DB_E4M3;
    p.e.act = v.act;
    const Plan plan = plan_forward(v.rows, v.n_in, v.n_out);
    float* partials = reinterpret_cast<float*>(arena.take(static_cast<size_t>(plan.partial_floats) * 4));
    if (count) return DB_OK;
    const db_status st = ops.copy_now(status, clear, stream);
    return st != DB_OK ? st : run_products(kForward, plan, &p, 1, partials, status, clear, stream);
}

struct LinearGradArgs {
    const void *dy, *x, *w, *z, *z_scale, *addend;
    long long dy_pitch, x_pitch, addend_pitch, rows;
    db_dtype z_dtype, grad_dtype;
    int n_in, n_out, act;
    void *dx, *dw, *dbias;
    long long dx_pitch;
};

int slab_count(long long rows, long long cols) {   // about four CTAs per SM, at least 32 rows each
    const long long across = cdiv(cols, 256);
    return static_cast<int>(std::max(1LL, std::min(cdiv(rows, 32), cdiv(4LL * sm_count(), across))));
}

db_status linear_backward(const LinearGradArgs& v, Arena& arena, cudaStream_t stream, bool aligned) {
    const bool count = !arena.base;
    int* status = reinterpret_cast<int*>(arena.base);
    bool clear = true;
    const void* off = aligned ? nullptr : reinterpret_cast<const void*>(2);
    const bool has_act = count || v.act != DB_ACT_NONE, want_bias = count || v.dbias, want_dw = count || v.dw, want_dx = count || v.dx;
    Matrix dz{static_cast<const bf16*>(v.dy), v.rows, v.n_out, v.dy_pitch};
    lg::BiasFold bias;
    Operands ops(arena);
    if (has_act || want_bias) {
        ActGradArgs a{};
        a.dy = static_cast<const bf16*>(v.dy); a.dy_pitch = v.dy_pitch;
        a.z = {const_cast<void*>(v.z), static_cast<uint8_t*>(const_cast<void*>(v.z_scale))};
        a.z_e4m3 = v.z_dtype == DB_E4M3;
        a.act = v.act;
        a.rows = v.rows; a.cols = v.n_out;
        if (has_act) {
            dz.pitch = (v.n_out + 31LL) / 32 * 32;
            a.dz = reinterpret_cast<bf16*>(arena.take(static_cast<size_t>(v.rows * dz.pitch) * 2));
            a.dz_pitch = dz.pitch;
            dz.p = a.dz;
        }
        const int slabs = slab_count(v.rows, v.n_out);
        a.slab_rows = static_cast<int>(cdiv(v.rows, slabs));
        const int used = a.slab_rows ? static_cast<int>(cdiv(v.rows, a.slab_rows)) : 1;
        if (want_bias) {
            a.sums_pitch = (v.n_out + 31LL) / 32 * 32;
            a.sums = reinterpret_cast<float*>(arena.take(static_cast<size_t>(slabs * a.sums_pitch) * 4));
        }
        if (!count) {
            a.clear_status = status;
            clear = false;
            Launch L(dim3(static_cast<unsigned>(cdiv(v.n_out, 256)), used), dim3(256), 0, stream);
            DB_CUDA_TRY(cudaLaunchKernelEx(&L.cfg, act_grad_fn(a.act, a.z_e4m3), a));
            if (want_bias) bias = {a.sums, a.sums_pitch, used, v.n_out, v.grad_dtype == DB_F32 ? 1 : 0, v.dbias};
            if (want_bias && !want_dx && !want_dw) {
                Launch F(dim3(static_cast<unsigned>(cdiv(v.n_out, 128))), dim3(128), 0, stream);
                DB_CUDA_TRY(cudaLaunchKernelEx(&F.cfg, bias_fold_kernel, bias));
            }
        }
    }
    if (count ? !aligned : !has_act && (want_dx || want_dw)) dz = ops.of(count ? off : v.dy, v.rows, v.n_out, count ? v.n_out : v.dy_pitch);
    const Size size_x{v.rows, v.n_in}, size_w{v.n_in, v.n_out};
    const Plan plan_x = plan_input_grad(v.rows, v.n_in, v.n_out, 1), plan_w = plan_weight_grad(&size_w, 1, v.rows);
    float* partials = reinterpret_cast<float*>(arena.take(static_cast<size_t>(std::max(plan_x.partial_floats, plan_w.partial_floats)) * 4));
    Product p, q;
    if (want_dx) {
        p.a[0] = dz;
        p.b[0] = ops.of(count ? off : v.w, v.n_in, v.n_out, count && aligned ? (v.n_out + 7) / 8 * 8 : v.n_out);
        p.size = size_x;
        p.e.out = v.dx; p.e.out_pitch = v.dx_pitch;
        p.e.addend = static_cast<const bf16*>(v.addend); p.e.addend_pitch = v.addend_pitch;
    }
    if (want_dw) {
        q.a[0] = ops.of(count ? off : v.x, v.rows, v.n_in, count ? (aligned ? (v.n_in + 7) / 8 * 8 : v.n_in) : v.x_pitch);
        q.b[0] = dz;
        q.size = size_w;
        q.e.out = v.dw; q.e.out_pitch = v.n_out;
        q.e.out_f32 = v.grad_dtype == DB_F32;
    }
    if (count) return DB_OK;
    db_status st = ops.copy_now(status, clear, stream);
    if (st == DB_OK && want_dx) st = run_products(kInputGrad, plan_x, &p, 1, partials, status, clear, stream, bias);
    if (st == DB_OK && want_dw) st = run_products(kWeightGrad, plan_w, &q, 1, partials, status, clear, stream, want_dx ? lg::BiasFold{} : bias);
    return st;
}

// ---------------------------------------------------------------------------------------------- gated block
struct GatedArgs {
    const void *dy, *x, *w_gate, *w_up, *w_down, *residual;
    long long dy_pitch, x_pitch, residual_pitch, rows;
    int width, hidden, act;
    void* y;                       // forward: y; backward: dx
    long long y_pitch;
    void *gate, *up, *gate_scale, *up_scale;
    db_dtype kept_dtype, grad_dtype;
    void *dw_gate, *dw_up, *dw_down;
};

db_status gated_forward(const GatedArgs& v, Arena& arena, cudaStream_t stream, bool aligned) {
    const bool count = !arena.base;
    int* status = reinterpret_cast<int*>(arena.base);
    bool clear = true;
    const void* off = aligned ? nullptr : reinterpret_cast<const void*>(2);
    Operands ops(arena);
    const long long h_pitch = (v.hidden + 31LL) / 32 * 32;
    bf16* h = reinterpret_cast<bf16*>(arena.take(static_cast<size_t>(v.rows * h_pitch) * 2));
    const auto pitch = [&](long long given, long long cols) { return !count ? given : aligned ? (cols + 7) / 8 * 8 : cols; };
    Product p, q;
    p.a[0] = ops.of(count ? off : v.x, v.rows, v.width, pitch(v.x_pitch, v.width));
    p.b[0] = ops.of(count ? off : v.w_gate, v.width, v.hidden, pitch(v.hidden, v.hidden));
    p.b[1] = ops.of(count ? off : v.w_up, v.width, v.hidden, pitch(v.hidden, v.hidden));
    p.size = {v.rows, v.hidden};
    p.e.out = h; p.e.out_pitch = h_pitch;
    p.e.kept[0] = {v.gate, static_cast<uint8_t*>(v.gate_scale)};
    p.e.kept[1] = {v.up, static_cast<uint8_t*>(v.up_scale)};
    p.e.kept_e4m3 = v.kept_dtype == DB_E4M3;
    p.e.act = v.act;
    q.a[0] = Matrix{h, v.rows, v.hidden, h_pitch};
    q.b[0] = ops.of(count ? off : v.w_down, v.hidden, v.width, pitch(v.width, v.width));
    q.size = {v.rows, v.width};
    q.e.out = v.y; q.e.out_pitch = v.y_pitch;
    q.e.addend = static_cast<const bf16*>(v.residual); q.e.addend_pitch = v.residual_pitch;
    const Plan a = plan_gated(v.rows, v.width, v.hidden), b = plan_forward(v.rows, v.hidden, v.width);
    float* partials = reinterpret_cast<float*>(arena.take(static_cast<size_t>(std::max(a.partial_floats, b.partial_floats)) * 4));
    if (count) return DB_OK;
    db_status st = ops.copy_now(status, clear, stream);
    if (st == DB_OK) st = run_products(kGated, a, &p, 1, partials, status, clear, stream);
    return st != DB_OK ? st : run_products(kForward, b, &q, 1, partials, status, clear, stream);
}

db_status gated_backward(const GatedArgs& v, Arena& arena, cudaStream_t stream, bool aligned) {
    const bool count = !arena.base;
    int* status = reinterpret_cast<int*>(arena.base);
    bool clear = true;
    const void* off = aligned ? nullptr : reinterpret_cast<const void*>(2);
    Operands ops(arena);
    const long long h_pitch = (v.hidden + 31LL) / 32 * 32;
    const size_t h_bytes = static_cast<size_t>(v.rows * h_pitch) * 2;
    bf16* h = reinterpret_cast<bf16*>(arena.take(h_bytes));
    bf16* d_gate = reinterpret_cast<bf16*>(arena.take(h_bytes));
    bf16* d_up = reinterpret_cast<bf16*>(arena.take(h_bytes));
    const auto pitch = [&](long long given, long long cols) { return !count ? given : aligned ? (cols + 7) / 8 * 8 : cols; };
    const bool want_dx = count || v.y, want_dw = count || v.dw_gate || v.dw_up || v.dw_down;
    const Matrix dy = ops.of(count ? off : v.dy, v.rows, v.width, pitch(v.dy_pitch, v.width));
    const Matrix mg{d_gate, v.rows, v.hidden, h_pitch}, mu{d_up, v.rows, v.hidden, h_pitch}, mh{h, v.rows, v.hidden, h_pitch};

    Product p, q, w[3];
    p.a[0] = dy;
    p.b[0] = ops.of(count ? off : v.w_down, v.hidden, v.width, pitch(v.width, v.width));
    p.size = {v.rows, v.hidden};
    p.e.out = h; p.e.out_pitch = h_pitch;
    p.e.d_gate = d_gate; p.e.d_up = d_up; p.e.d_pitch = h_pitch;
    p.e.kept[0] = {v.gate, static_cast<uint8_t*>(v.gate_scale)};
    p.e.kept[1] = {v.up, static_cast<uint8_t*>(v.up_scale)};
    p.e.kept_e4m3 = v.kept_dtype == DB_E4M3;
    p.e.act = v.act;
    const Plan plan_p = plan_gated_grad(v.rows, v.width, v.hidden);

    if (want_dx) {
        q.a[0] = mg; q.a[1] = mu;
        q.b[0] = ops.of(count ? off : v.w_gate, v.width, v.hidden, pitch(v.hidden, v.hidden));
        q.b[1] = ops.of(count ? off : v.w_up, v.width, v.hidden, pitch(v.hidden, v.hidden));
        q.sources = 2;
        q.size = {v.rows, v.width};
        q.e.out = v.y; q.e.out_pitch = v.y_pitch;
        q.e.addend = static_cast<const bf16*>(v.residual); q.e.addend_pitch = v.residual_pitch;
    }
    const Plan plan_q = want_dx ? plan_input_grad(v.rows, v.width, v.hidden, 2) : Plan{};

    int n = 0;
    Size sizes[3];
    if (want_dw) {
        const bool x_used = count || v.dw_gate || v.dw_up;
        const Matrix x = x_used ? ops.of(count ? off : v.x, v.rows, v.width, pitch(v.x_pitch, v.width)) : Matrix{};
        const auto add = [&](const Matrix& a, const Matrix& b, void* out) {
            if (!count && !out) return;
            w[n].a[0] = a; w[n].b[0] = b;
            w[n].size = {a.cols, b.cols};
            w[n].e.out = out; w[n].e.out_pitch = b.cols;
            w[n].e.out_f32 = v.grad_dtype == DB_F32;
            sizes[n] = w[n].size;
            ++n;
        };
        add(x, mg, v.dw_gate);
        add(x, mu, v.dw_up);
        add(mh, dy, v.dw_down);
    }
    long long floats = std::max(plan_p.partial_floats, plan_q.partial_floats);
    // which weight gradients a call wants decides how its reduction is split: room for any choice
    if (count) {
        const Size up{v.width, v.hidden}, down{v.hidden, v.width};
        const Size choices[5][3] = {{up}, {down}, {up, up}, {up, down}, {up, up, down}};
        const int counts[5] = {1, 1, 2, 2, 3};
        for (int i = 0; i < 5; ++i) floats = std::max(floats, plan_weight_grad(choices[i], counts[i], v.rows).partial_floats);
    }
    const Plan plan_w = plan_weight_grad(sizes, n, v.rows);
    floats = std::max(floats, plan_w.partial_floats);
    float* partials = reinterpret_cast<float*>(arena.take(static_cast<size_t>(floats) * 4));
    if (count) return DB_OK;
    db_status st = ops.copy_now(status, clear, stream);
    if (st == DB_OK) st = run_products(kGatedGrad, plan_p, &p, 1, partials, status, clear, stream);
    if (st == DB_OK && want_dx) st = run_products(kInputGrad, plan_q, &q, 1, partials, status, clear, stream);
    if (st == DB_OK && n) st = run_products(kWeightGrad, plan_w, w, n, partials, status, clear, stream);
    return st;
}

}  // namespace
}  // namespace dynbatch

// ---------------------------------------------------------------------------------------------- entry points
extern "C" size_t db_linear_workspace_bytes(int64_t rows, int32_t n_in, int32_t n_out, int32_t aligned) {
    using namespace dynbatch;
    if (!valid_size(rows, n_in, n_out)) return 0;
    LinearArgs v{};
    v.rows = rows; v.n_in = n_in; v.n_out = n_out;
    Arena arena(nullptr);
    linear_forward(v, arena, nullptr, aligned && n_in % 8 == 0 && n_out % 8 == 0);
    return arena.used;
}

extern "C" db_status db_linear(const void* x, int64_t x_pitch, const void* w, const void* bias, const void* residual,
                               int64_t residual_pitch, db_activation act, int64_t rows, int32_t n_in, int32_t n_out, void* y,
                               int64_t y_pitch, void* z, void* z_scale, db_dtype z_dtype, void* workspace,
                               size_t workspace_bytes, void* cuda_stream) {
    using namespace dynbatch;
    if (!w || !workspace) return DB_ERR_NULL;
    if (!valid_size(rows, n_in, n_out)) return DB_ERR_ARG;
    if (rows > 0 && (!x || !y)) return DB_ERR_NULL;
    if (!valid_act(act)) return DB_ERR_UNSUPPORTED;
    if (z && z_dtype != DB_BF16 && z_dtype != DB_E4M3) return DB_ERR_UNSUPPORTED;
    if (z && z_dtype == DB_E4M3 && !z_scale) return DB_ERR_NULL;
    if (!valid_pitch(x, n_in, x_pitch) || !valid_pitch(y, n_out, y_pitch) || !valid_pitch(residual, n_out, residual_pitch)) return DB_ERR_ARG;
    if (odd_address(x, 2) || odd_address(w, 2) || odd_address(bias, 2) || odd_address(residual, 2) || odd_address(y, 2) ||
        (z && z_dtype == DB_BF16 && odd_address(z, 2)) || odd_address(workspace, 256))
        return DB_ERR_ARG;
    const bool e4m3 = z && z_dtype == DB_E4M3;
    const bool in_place = residual == y && residual_pitch == y_pitch;
    const Extent touched[] = {
        matrix(x, rows, n_in, x_pitch, 2, false), matrix(w, n_in, n_out, n_out, 2, false),
        block(bias, 2LL * n_out, false), matrix(in_place ? nullptr : residual, rows, n_out, residual_pitch, 2, false),
        matrix(y, rows, n_out, y_pitch, 2, true), block(z, z ? rows * n_out * kept_size(z_dtype) : 0, true),
        block(e4m3 ? z_scale : nullptr, rows * scales_of(n_out), true), block(workspace, static_cast<long long>(workspace_bytes), true)};
    if (overlaps(touched)) return DB_ERR_ARG;
    const bool aligned = on_grid(x, x_pitch) && on_grid(w, n_out);
    LinearArgs v{x, w, bias, residual, x_pitch, residual_pitch, rows, n_in, n_out, act, y, y_pitch, z, z_scale, z_dtype};
    Arena need(nullptr);
    linear_forward(v, need, nullptr, aligned);
    if (workspace_bytes < need.used) return DB_ERR_ARG;
    if (rows == 0) return zero(workspace, 4, static_cast<cudaStream_t>(cuda_stream));
    Arena arena(workspace);
    return linear_forward(v, arena, static_cast<cudaStream_t>(cuda_stream), aligned);
}

extern "C" size_t db_linear_grad_workspace_bytes(int64_t rows, int32_t n_in, int32_t n_out, int32_t aligned) {
    using namespace dynbatch;
    if (!valid_size(rows, n_in, n_out)) return 0;
    LinearGradArgs v{};
    v.rows = rows; v.n_in = n_in; v.n_out = n_out;
    Arena arena(nullptr);
    linear_backward(v, arena, nullptr, aligned && n_in % 8 == 0 && n_out % 8 == 0);
    return arena.used;
}

extern "C" db_status db_linear_grad(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, const void* w,
                                    const void* z, const void* z_scale, db_dtype z_dtype, db_activation act, int64_t rows,
                                    int32_t n_in, int32_t n_out, void* dx, int64_t dx_pitch, const void* dx_addend,
                                    int64_t dx_addend_pitch, void* dw, void* dbias, db_dtype grad_dtype, void* workspace,
                                    size_t workspace_bytes, void* cuda_stream) {
    using namespace dynbatch;
    if (!workspace || (!dx && !dw && !dbias)) return DB_ERR_NULL;
    if (!valid_size(rows, n_in, n_out)) return DB_ERR_ARG;
    if (!valid_act(act)) return DB_ERR_UNSUPPORTED;
    if (grad_dtype != DB_F32 && grad_dtype != DB_BF16) return DB_ERR_UNSUPPORTED;
    if (act != DB_ACT_NONE && z_dtype != DB_BF16 && z_dtype != DB_E4M3) return DB_ERR_UNSUPPORTED;
    if (rows > 0) {
        if (!dy || (dw && !x) || (dx && !w)) return DB_ERR_NULL;
        if (act != DB_ACT_NONE && (!z || (z_dtype == DB_E4M3 && !z_scale))) return DB_ERR_NULL;
    }
    if (dx_addend && !dx) return DB_ERR_ARG;
    if (!valid_pitch(dy, n_out, dy_pitch) || !valid_pitch(dw ? x : nullptr, n_in, x_pitch) || !valid_pitch(dx, n_in, dx_pitch) ||
        !valid_pitch(dx_addend, n_in, dx_addend_pitch))
        return DB_ERR_ARG;
    const bool with_z = act != DB_ACT_NONE;
    const int g = grad_dtype == DB_F32 ? 4 : 2;
    if (odd_address(dy, 2) || odd_address(x, 2) || odd_address(w, 2) || (with_z && z_dtype == DB_BF16 && odd_address(z, 2)) ||
        odd_address(dx, 2) || odd_address(dx_addend, 2) || odd_address(dw, g) || odd_address(dbias, g) || odd_address(workspace, 256))
        return DB_ERR_ARG;
    const bool in_place = dx_addend == dx && dx_addend_pitch == dx_pitch;
    const Extent touched[] = {
        matrix(dy, rows, n_out, dy_pitch, 2, false), matrix(dw ? x : nullptr, rows, n_in, x_pitch, 2, false),
        matrix(dx ? w : nullptr, n_in, n_out, n_out, 2, false),
        block(with_z ? z : nullptr, rows * n_out * kept_size(z_dtype), false),
        block(with_z && z_dtype == DB_E4M3 ? z_scale : nullptr, rows * scales_of(n_out), false),
        matrix(in_place ? nullptr : dx_addend, rows, n_in, dx_addend_pitch, 2, false),
        matrix(dx, rows, n_in, dx_pitch, 2, true), block(dw, static_cast<long long>(n_in) * n_out * g, true),
        block(dbias, static_cast<long long>(n_out) * g, true), block(workspace, static_cast<long long>(workspace_bytes), true)};
    if (overlaps(touched)) return DB_ERR_ARG;
    const bool aligned = (with_z || (!dx && !dw) || on_grid(dy, dy_pitch)) && (!dw || on_grid(x, x_pitch)) && (!dx || on_grid(w, n_out));
    LinearGradArgs v{dy, x, w, z, z_scale, dx_addend, dy_pitch, x_pitch, dx_addend_pitch, rows, z_dtype, grad_dtype,
                     n_in, n_out, act, dx, dw, dbias, dx_pitch};
    Arena need(nullptr);
    linear_backward(v, need, nullptr, aligned);
    if (workspace_bytes < need.used) return DB_ERR_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {             // a batch without rows has zero gradients
        db_status st = zero(workspace, 4, stream);
        if (st == DB_OK) st = zero(dw, static_cast<long long>(n_in) * n_out * g, stream);
        return st != DB_OK ? st : zero(dbias, static_cast<long long>(n_out) * g, stream);
    }
    Arena arena(workspace);
    return linear_backward(v, arena, stream, aligned);
}

extern "C" size_t db_gated_ffn_workspace_bytes(int64_t rows, int32_t width, int32_t hidden, int32_t aligned) {
    using namespace dynbatch;
    if (!valid_size(rows, width, hidden)) return 0;
    GatedArgs v{};
    v.rows = rows; v.width = width; v.hidden = hidden;
    Arena arena(nullptr);
    gated_forward(v, arena, nullptr, aligned && width % 8 == 0 && hidden % 8 == 0);
    return arena.used;
}

extern "C" db_status db_gated_ffn(const void* x, int64_t x_pitch, const void* w_gate, const void* w_up, const void* w_down,
                                  const void* residual, int64_t residual_pitch, db_activation act, int64_t rows, int32_t width,
                                  int32_t hidden, void* y, int64_t y_pitch, void* gate, void* up, void* gate_scale,
                                  void* up_scale, db_dtype kept_dtype, void* workspace, size_t workspace_bytes,
                                  void* cuda_stream) {
    using namespace dynbatch;
    if (!w_gate || !w_up || !w_down || !workspace) return DB_ERR_NULL;
    if (!valid_size(rows, width, hidden)) return DB_ERR_ARG;
    if (rows > 0 && (!x || !y)) return DB_ERR_NULL;
    if (!valid_act(act)) return DB_ERR_UNSUPPORTED;
    if (!gate != !up) return DB_ERR_NULL;                         // both or neither
    if (gate && kept_dtype != DB_BF16 && kept_dtype != DB_E4M3) return DB_ERR_UNSUPPORTED;
    const bool e4m3 = gate && kept_dtype == DB_E4M3;
    if (e4m3 && (!gate_scale || !up_scale)) return DB_ERR_NULL;
    if (!valid_pitch(x, width, x_pitch) || !valid_pitch(y, width, y_pitch) || !valid_pitch(residual, width, residual_pitch)) return DB_ERR_ARG;
    const bool kept16 = gate && !e4m3;
    if (odd_address(x, 2) || odd_address(w_gate, 2) || odd_address(w_up, 2) || odd_address(w_down, 2) || odd_address(residual, 2) ||
        odd_address(y, 2) || (kept16 && (odd_address(gate, 2) || odd_address(up, 2))) || odd_address(workspace, 256))
        return DB_ERR_ARG;
    const long long weight = 2LL * width * hidden, kept = gate ? rows * hidden * kept_size(kept_dtype) : 0, scales = rows * scales_of(hidden);
    const bool in_place = residual == y && residual_pitch == y_pitch;
    const Extent touched[] = {
        matrix(x, rows, width, x_pitch, 2, false), block(w_gate, weight, false), block(w_up, weight, false), block(w_down, weight, false),
        matrix(in_place ? nullptr : residual, rows, width, residual_pitch, 2, false),
        matrix(y, rows, width, y_pitch, 2, true), block(gate, kept, true), block(up, kept, true),
        block(e4m3 ? gate_scale : nullptr, scales, true), block(e4m3 ? up_scale : nullptr, scales, true),
        block(workspace, static_cast<long long>(workspace_bytes), true)};
    if (overlaps(touched)) return DB_ERR_ARG;
    const bool aligned = on_grid(x, x_pitch) && on_grid(w_gate, hidden) && on_grid(w_up, hidden) && on_grid(w_down, width);
    GatedArgs v{};
    v.x = x; v.x_pitch = x_pitch; v.w_gate = w_gate; v.w_up = w_up; v.w_down = w_down;
    v.residual = residual; v.residual_pitch = residual_pitch; v.act = act;
    v.rows = rows; v.width = width; v.hidden = hidden; v.y = y; v.y_pitch = y_pitch;
    v.gate = gate; v.up = up; v.gate_scale = gate_scale; v.up_scale = up_scale; v.kept_dtype = kept_dtype;
    Arena need(nullptr);
    gated_forward(v, need, nullptr, aligned);
    if (workspace_bytes < need.used) return DB_ERR_ARG;
    if (rows == 0) return zero(workspace, 4, static_cast<cudaStream_t>(cuda_stream));
    Arena arena(workspace);
    return gated_forward(v, arena, static_cast<cudaStream_t>(cuda_stream), aligned);
}

extern "C" size_t db_gated_ffn_grad_workspace_bytes(int64_t rows, int32_t width, int32_t hidden, int32_t aligned) {
    using namespace dynbatch;
    if (!valid_size(rows, width, hidden)) return 0;
    GatedArgs v{};
    v.rows = rows; v.width = width; v.hidden = hidden;
    Arena arena(nullptr);
    gated_backward(v, arena, nullptr, aligned && width % 8 == 0 && hidden % 8 == 0);
    return arena.used;
}

extern "C" db_status db_gated_ffn_grad(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, const void* w_gate,
                                       const void* w_up, const void* w_down, const void* gate, const void* up,
                                       const void* gate_scale, const void* up_scale, db_dtype kept_dtype, db_activation act,
                                       int64_t rows, int32_t width, int32_t hidden, void* dx, int64_t dx_pitch,
                                       const void* dx_addend, int64_t dx_addend_pitch, void* dw_gate, void* dw_up,
                                       void* dw_down, db_dtype grad_dtype, void* workspace, size_t workspace_bytes,
                                       void* cuda_stream) {
    using namespace dynbatch;
    if (!workspace || !w_down || (!dx && !dw_gate && !dw_up && !dw_down)) return DB_ERR_NULL;
    if (!valid_size(rows, width, hidden)) return DB_ERR_ARG;
    if (!valid_act(act)) return DB_ERR_UNSUPPORTED;
    if (grad_dtype != DB_F32 && grad_dtype != DB_BF16) return DB_ERR_UNSUPPORTED;
    if (kept_dtype != DB_BF16 && kept_dtype != DB_E4M3) return DB_ERR_UNSUPPORTED;
    const bool e4m3 = kept_dtype == DB_E4M3, needs_x = dw_gate || dw_up;
    if (rows > 0) {
        if (!dy || !gate || !up || (e4m3 && (!gate_scale || !up_scale))) return DB_ERR_NULL;
        if ((needs_x && !x) || (dx && (!w_gate || !w_up))) return DB_ERR_NULL;
    }
    if (dx_addend && !dx) return DB_ERR_ARG;
    if (!valid_pitch(dy, width, dy_pitch) || !valid_pitch(needs_x ? x : nullptr, width, x_pitch) || !valid_pitch(dx, width, dx_pitch) ||
        !valid_pitch(dx_addend, width, dx_addend_pitch))
        return DB_ERR_ARG;
    const int g = grad_dtype == DB_F32 ? 4 : 2;
    if (odd_address(dy, 2) || odd_address(x, 2) || odd_address(w_gate, 2) || odd_address(w_up, 2) || odd_address(w_down, 2) ||
        (!e4m3 && (odd_address(gate, 2) || odd_address(up, 2))) || odd_address(dx, 2) || odd_address(dx_addend, 2) ||
        odd_address(dw_gate, g) || odd_address(dw_up, g) || odd_address(dw_down, g) || odd_address(workspace, 256))
        return DB_ERR_ARG;
    const long long weight = 2LL * width * hidden, grad = static_cast<long long>(g) * width * hidden;
    const long long kept = rows * hidden * kept_size(kept_dtype), scales = rows * scales_of(hidden);
    const bool in_place = dx_addend == dx && dx_addend_pitch == dx_pitch;
    const Extent touched[] = {
        matrix(dy, rows, width, dy_pitch, 2, false), matrix(needs_x ? x : nullptr, rows, width, x_pitch, 2, false),
        block(dx ? w_gate : nullptr, weight, false), block(dx ? w_up : nullptr, weight, false), block(w_down, weight, false),
        block(gate, kept, false), block(up, kept, false), block(e4m3 ? gate_scale : nullptr, scales, false), block(e4m3 ? up_scale : nullptr, scales, false),
        matrix(in_place ? nullptr : dx_addend, rows, width, dx_addend_pitch, 2, false),
        matrix(dx, rows, width, dx_pitch, 2, true), block(dw_gate, grad, true), block(dw_up, grad, true), block(dw_down, grad, true),
        block(workspace, static_cast<long long>(workspace_bytes), true)};
    if (overlaps(touched)) return DB_ERR_ARG;
    const bool aligned = on_grid(dy, dy_pitch) && (!needs_x || on_grid(x, x_pitch)) && on_grid(w_down, width) &&
                         (!dx || (on_grid(w_gate, hidden) && on_grid(w_up, hidden)));
    GatedArgs v{};
    v.dy = dy; v.dy_pitch = dy_pitch; v.x = x; v.x_pitch = x_pitch;
    v.w_gate = w_gate; v.w_up = w_up; v.w_down = w_down;
    v.residual = dx_addend; v.residual_pitch = dx_addend_pitch; v.act = act;
    v.rows = rows; v.width = width; v.hidden = hidden; v.y = dx; v.y_pitch = dx_pitch;
    v.gate = const_cast<void*>(gate); v.up = const_cast<void*>(up);
    v.gate_scale = const_cast<void*>(gate_scale); v.up_scale = const_cast<void*>(up_scale);
    v.kept_dtype = kept_dtype; v.grad_dtype = grad_dtype;
    v.dw_gate = dw_gate; v.dw_up = dw_up; v.dw_down = dw_down;
    Arena need(nullptr);
    gated_backward(v, need, nullptr, aligned);
    if (workspace_bytes < need.used) return DB_ERR_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {
        db_status st = zero(workspace, 4, stream);
        for (void* p : {dw_gate, dw_up, dw_down})
            if (st == DB_OK) st = zero(p, grad, stream);
        return st;
    }
    Arena arena(workspace);
    return gated_backward(v, arena, stream, aligned);
}

extern "C" db_status db_bench_layer_plan(db_bench_layer_product product, int64_t rows, int32_t n_in, int32_t n_out,
                                         int32_t* ctas_per_tile, int32_t* tile_columns, int32_t* pieces) {
    using namespace dynbatch;
    if (!ctas_per_tile || !tile_columns || !pieces) return DB_ERR_NULL;
    if (!valid_size(rows, n_in, n_out) || rows == 0) return DB_ERR_ARG;
    const Size up{n_in, n_out}, down{n_out, n_in}, all[3] = {up, up, down};
    Plan p;
    switch (product) {
        case DB_BENCH_LINEAR_Y: p = plan_forward(rows, n_in, n_out); break;
        case DB_BENCH_LINEAR_DX: p = plan_input_grad(rows, n_in, n_out, 1); break;
        case DB_BENCH_LINEAR_DW: p = plan_weight_grad(&up, 1, rows); break;
        case DB_BENCH_GATED_H: p = plan_gated(rows, n_in, n_out); break;
        case DB_BENCH_GATED_Y: p = plan_forward(rows, n_out, n_in); break;
        case DB_BENCH_GATED_DH: p = plan_gated_grad(rows, n_in, n_out); break;
        case DB_BENCH_GATED_DX: p = plan_input_grad(rows, n_in, n_out, 2); break;
        case DB_BENCH_GATED_DW: p = plan_weight_grad(all, 3, rows); break;
        default: return DB_ERR_UNSUPPORTED;
    }
    *ctas_per_tile = kShapes[p.shape].cg;
    *tile_columns = kShapes[p.shape].bn;
    *pieces = p.splits;
    return DB_OK;
}
