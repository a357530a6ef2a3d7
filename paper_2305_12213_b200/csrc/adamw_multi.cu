// AdamW over a list of parameter tensors for K workers' batch-weighted gradients, moments in 32 or 8 bits, with
// optional clipping by the global norm; and that norm alone.  A plan holds records in device memory, as for the
// momentum step over a list; a step is one launch (and one or two folds where it leaves the norm), two to four when it
// clips: norm of the aggregate, on long lists one or two folds, update.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <exception>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "adamw_kernels.cuh"
#include "common.h"

namespace dynbatch {
namespace {

using namespace adamw;

size_t round256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
long long blocks_of(long long n) { return n / kWarpElems + (n % kWarpElems != 0); }
size_t grad_bytes(db_dtype dt) { return dt == DB_F32 ? 4 : 2; }

// The fold sums up to kFoldPer partials with one CTA; beyond that a first stage of CTAs takes kFoldPer each.
constexpr int kFoldPer = 8192;

// CTA steps (kSpan elements) in the list; false if a size is negative or there are more than a grid takes.
bool count_spans(const int64_t* sizes, int32_t T, long long* spans) {
    long long sum = 0;
    for (int32_t t = 0; t < T; ++t) {
        if (sizes[t] < 0) return false;
        sum += sizes[t] / kSpan + (sizes[t] % kSpan != 0);
        if (sum > 0x3fffffffLL) return false;
    }
    *spans = sum;
    return true;
}

// Whether a clipped step lets the norm kernel leave the aggregate (4 bytes written, 4 read for each element)
// instead of reading the K gradients a second time.
bool stages(int K, db_dtype dt) { return static_cast<size_t>(K) * grad_bytes(dt) > 8; }

// Elements of an 8-bit step's record, in CTA steps: one for short lists, two from 2000 steps on (a ring is filled once
// for both), and up to eight as long as 2400 records are left (16 for each of 148 SMs).  A longer run fills its ring
// less often, but spreads the CTAs' streams and fills the last wave less evenly (us; 5M parameters, one bf16 gradient,
// 1, 2, 3 steps: 22.9, 18.5, 17.7; 10M, four fp32, 2, 4, 6: 48.2, 52.3, 50.0; 25M, four fp32, 5, 8: 112.9, 120.3; 470M,
// one bf16, clipped, 4, 8, 16: 1536, 1487, 1521).  One step against two about 2000 of them (replayed, over buffers beyond
// the L2): at 600 steps one bf16 gradient 7.3 and 7.0, three fp32 9.3 and 10.0, eight bf16 10.7 and 11.4; at 1000 10.8 and
// 9.5, 13.8 and 12.7, 15.8 and 14.6; at 2000 18.6 and 15.5, 23.5 and 22.2, 27.1 and 25.7: two would do from 1000 on.
int run_of(long long spans) {
    const long long least = spans < 2000 ? 1 : 2;
    return kSpan * static_cast<int>(std::min<long long>(8, std::max(least, spans / 2400)));
}

// One kind of records: `run` elements each, `stride` words apart.
struct Records {
    int run, stride;
    long long count;
    size_t at;
};

Records records_of(const int64_t* sizes, int32_t T, int run, int words, size_t* end) {
    Records r{run, (words + 1) & ~1, 0, *end};                      // an even stride: records stay 16-byte aligned
    for (int32_t t = 0; t < T; ++t) r.count += sizes[t] / run + (sizes[t] % run != 0);
    *end += round256(8 * static_cast<size_t>(r.stride) * static_cast<size_t>(r.count));
    return r;
}

struct Layout {
    Records step, norm;
    size_t partials, sums, scalars, staged, end;                    // scalars: ticket, clipping factor
};

// Elements of a norm record: as much as the kernel for all K workers has in flight at once.
template <typename GT>
int norm_run(int K) { return kSpan * norm_batch<GT>(K <= 1 ? 1 : K <= 2 ? 2 : K <= 4 ? 4 : 8); }     // as in pick_norm

// step: records of the optimizer step (state8: several CTA steps each); norm: records of the norm kernel.
bool make_layout(int32_t K, db_dtype dt, bool state8, const int64_t* sizes, int32_t T, bool step, bool norm, Layout* L) {
    long long spans;
    if (!count_spans(sizes, T, &spans)) return false;
    L->end = 0;
    L->step = L->norm = Records{};
    if (step) L->step = records_of(sizes, T, state8 ? run_of(spans) : kSpan, kRecGrads + K, &L->end);
    if (norm) L->norm = records_of(sizes, T, dt == DB_F32 ? norm_run<float>(K) : norm_run<__nv_bfloat16>(K), kNormGrads + K, &L->end);
    const size_t n = static_cast<size_t>(std::max<long long>(1, std::max(L->step.count, 2 * L->norm.count)));
    L->partials = L->end;
    L->sums = L->partials + round256(8 * n);
    L->scalars = L->sums + round256(8 * (n / kFoldPer + 1));
    L->staged = L->scalars + 256;
    size_t staged = 0;
    if (step && norm && stages(K, dt))
        for (int32_t t = 0; t < T; ++t) staged += static_cast<size_t>(blocks_of(sizes[t])) * kWarpElems * 4;
    L->end = L->staged + staged;
    return true;
}

struct Range {
    uintptr_t begin, end;
    bool operator<(const Range& o) const { return begin < o.begin; }
};

// Buffers that a step writes may not overlap one another, nor a gradient one of them.
bool overlaps(std::vector<Range>& written, const std::vector<Range>& read) {
    std::sort(written.begin(), written.end());
    for (size_t i = 1; i < written.size(); ++i)
        if (written[i].begin < written[i - 1].end) return true;
    for (const Range& r : read) {
        const auto it = std::lower_bound(written.begin(), written.end(), Range{r.end, 0});   // the first that begins at or behind r's end
        if (it != written.begin() && std::prev(it)->end > r.begin) return true;
    }
    return false;
}

void add_range(std::vector<Range>& v, const void* p, long long n, size_t elem) {
    if (n > 0 && p) v.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + static_cast<size_t>(n) * elem});
}

long long word(const void* p) { return static_cast<long long>(reinterpret_cast<uintptr_t>(p)); }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// Uploads records and the cleared ticket and waits for it: plan creation is not on the hot path, and not possible
// in a capture.
db_status upload(const Layout& L, const std::vector<long long>& step, const std::vector<long long>& norm, char* table,
                 cudaStream_t stream, const char* where) {
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (stream) DB_CUDA_TRY(cudaStreamIsCapturing(stream, &capture));
    if (capture != cudaStreamCaptureStatusNone) {
        record_message("a plan cannot be created while its stream is being captured");
        return DB_ERR_UNSUPPORTED;
    }
    cudaError_t err = cudaMemsetAsync(table + L.scalars, 0, 256, stream);
    if (err == cudaSuccess && !step.empty())
        err = cudaMemcpyAsync(table + L.step.at, step.data(), 8 * step.size(), cudaMemcpyHostToDevice, stream);
    if (err == cudaSuccess && !norm.empty())
        err = cudaMemcpyAsync(table + L.norm.at, norm.data(), 8 * norm.size(), cudaMemcpyHostToDevice, stream);
    // the host vectors go away when the caller returns
    const cudaError_t done = cudaStreamSynchronize(stream);
    if (err == cudaSuccess) err = done;
    return err == cudaSuccess ? DB_OK : record_cuda_error(err, where);
}

// Both halves of a packed pair.
unsigned long long pair_of(float x) {
    uint32_t bits;
    __builtin_memcpy(&bits, &x, 4);
    return static_cast<unsigned long long>(bits) << 32 | bits;
}

// The workers of a call: weights of those with samples.  DB_ERR_ARG if a batch is negative or all are empty.
db_status set_workers(const int32_t* b, int K, Source* s) {
    long long total = 0;
    for (int k = 0; k < K; ++k) {
        if (b[k] < 0) return DB_ERR_ARG;
        total += b[k];
    }
    if (total <= 0) return DB_ERR_ARG;
    s->one = pair_of(1.0f);
    s->K = 0;
    for (int k = 0; k < K; ++k) {
        if (b[k] == 0) continue;
        s->lambda[s->K] = pair_of(static_cast<float>(static_cast<double>(b[k]) / static_cast<double>(total)));
        s->worker[s->K++] = static_cast<unsigned char>(k);
    }
    return DB_OK;
}

// Every kernel may be scheduled while its predecessor in the stream still runs; it waits before its first access.
template <typename... Params, typename... Args>
cudaError_t launch(void (*fn)(Params...), long long grid, int block, size_t shared, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1]{};
    cfg.gridDim = dim3(static_cast<unsigned int>(grid));
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, args...);
}

db_status launch_fold(const Layout& L, char* table, long long n, float* norm, float* factor, float max_norm, cudaStream_t stream) {
    const double* partials = reinterpret_cast<const double*>(table + L.partials);
    double* sums = reinterpret_cast<double*>(table + L.sums);
    if (n > kFoldPer) {
        const long long stage = (n + kFoldPer - 1) / kFoldPer;
        DB_CUDA_TRY(launch(fold_kernel, stage, 1024, 0, stream, partials, n, kFoldPer, sums, static_cast<float*>(nullptr),
                           static_cast<float*>(nullptr), 0.0f));
        partials = sums;
        n = stage;
    }
    DB_CUDA_TRY(launch(fold_kernel, 1, n > 256 ? 1024 : 256, 0, stream, partials, n, static_cast<int>(n),
                       static_cast<double*>(nullptr), norm, factor, max_norm));
    return DB_OK;
}

using NormFn = void (*)(const NormArgs);
template <typename GT, bool LAST>
NormFn pick_norm(int K) {
    if (K <= 1) return grad_norm_kernel<GT, 1, false, LAST>;
    if (K <= 2) return grad_norm_kernel<GT, 2, false, LAST>;
    if (K <= 4) return grad_norm_kernel<GT, 4, false, LAST>;
    if (K <= 8) return grad_norm_kernel<GT, 8, false, LAST>;
    if constexpr (sizeof(GT) == 2)
        if (K <= 16) return grad_norm_kernel<GT, 16, false, LAST>;
    return grad_norm_kernel<GT, 8, true, LAST>;
}

// Norm (and aggregate, and clipping factor) of a plan's gradients.  left: where the caller adds the partials itself if
// they are few, their number (0: done here).
db_status launch_norm(const Layout& L, char* table, db_dtype dt, int workers, Source src, float* norm, float* factor, float max_norm,
                      int* left, cudaStream_t stream) {
    NormArgs a{};
    a.src = src;
    a.src.recs = reinterpret_cast<const long long*>(table + L.norm.at);
    a.src.records = L.norm.count;
    a.src.stride = L.norm.stride;
    a.partials = reinterpret_cast<double*>(table + L.partials);
    a.ticket = reinterpret_cast<unsigned int*>(table + L.scalars);
    a.norm = norm;
    a.factor = factor;
    a.max_norm = max_norm;
    const long long grid = 2 * L.norm.count;
    // The norm kernel's last CTA adds the partials on grids of about a wave, which saves a launch where the host bounds the
    // call: norms of 20k and 1M elements, one fp32 gradient, 5.1 and 5.4 us a call against 7.0 and 7.1 with a fold kernel;
    // 1M, three gradients, 6.3 against 7.0; at the limit (4.5M, one; 1.1M, four) 7.5 against 7.3 and 8.2 against 7.6.  On the
    // device alone (replayed) the fold kernel takes 0.4 to 1.1 us less at all of these; beyond the limit the last CTA costs
    // another 2 to 5.
    const bool leave = left && grid <= kFoldInStep, last = !leave && grid <= 8 * sm_count();
    if (left) *left = leave ? static_cast<int>(grid) : 0;
    // by the plan's workers, not the call's: the records are made for that kernel
    const NormFn fn = dt == DB_F32 ? (last ? pick_norm<float, true>(workers) : pick_norm<float, false>(workers))
                                   : (last ? pick_norm<__nv_bfloat16, true>(workers) : pick_norm<__nv_bfloat16, false>(workers));
    DB_CUDA_TRY(launch(fn, grid, kNormThreads, 0, stream, a));
    return leave || last ? DB_OK : launch_fold(L, table, grid, norm, factor, max_norm, stream);
}

using StepFn = void (*)(const StepArgs);
template <typename GT, bool CLIP, bool NORM>
StepFn pick_workers(int K) {
    if (K <= 1) return adamw_kernel<GT, 1, false, CLIP, NORM>;
    if (K <= 2) return adamw_kernel<GT, 2, false, CLIP, NORM>;
    if (K <= 4) return adamw_kernel<GT, 4, false, CLIP, NORM>;
    if (K <= 8) return adamw_kernel<GT, 8, false, CLIP, NORM>;
    if constexpr (sizeof(GT) == 2)
        if (K <= 16) return adamw_kernel<GT, 16, false, CLIP, NORM>;
    return adamw_kernel<GT, sizeof(GT) == 2 ? 8 : 4, true, CLIP, NORM>;
}
template <typename GT>
StepFn pick_step(int K, bool clip, bool norm) {
    if (clip) return pick_workers<GT, true, false>(K);
    return norm ? pick_workers<GT, false, true>(K) : pick_workers<GT, false, false>(K);
}

// 8-bit moments: the kernel for K workers and the shared memory of its ring.
template <typename GT, bool CLIP, bool NORM>
StepFn pick_workers8(int K, size_t* shared) {
    *shared = K <= 1 ? Ring<GT, 1>::kBytes : K <= 2 ? Ring<GT, 2>::kBytes : Ring<GT, 4>::kBytes;       // as for 4, so for 8
    static_assert(Ring<GT, 4>::kBytes == Ring<GT, 8>::kBytes, "items do not depend on the number of workers beyond 2");
    if (K <= 1) return adamw8_kernel<GT, 1, false, CLIP, NORM>;
    if (K <= 2) return adamw8_kernel<GT, 2, false, CLIP, NORM>;
    if (K <= 4) return adamw8_kernel<GT, 4, false, CLIP, NORM>;
    if (K <= 8) return adamw8_kernel<GT, 8, false, CLIP, NORM>;
    return adamw8_kernel<GT, 8, true, CLIP, NORM>;
}
template <typename GT>
StepFn pick_step8(int K, bool clip, bool norm, size_t* shared) {
    if (clip) return pick_workers8<GT, true, false>(K, shared);
    return norm ? pick_workers8<GT, false, true>(K, shared) : pick_workers8<GT, false, false>(K, shared);
}

// The 8-bit kernels that a plan may launch may use as much shared memory as their rings take (per device: at creation).
template <typename GT>
cudaError_t allow_shared() {
    cudaError_t err = cudaSuccess;
    for (int K : {1, 2, 4, 8, 9})
        for (int mode = 0; err == cudaSuccess && mode < 3; ++mode) {
            size_t shared;
            const StepFn fn = pick_step8<GT>(K, mode == 1, mode == 2, &shared);
            err = cudaFuncSetAttribute(reinterpret_cast<const void*>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(shared));
        }
    return err;
}
db_status allow_shared(db_dtype dt) {
    cudaError_t err = allow_shared<float>();                  // a staged aggregate is fp32, whatever the gradients are
    if (err == cudaSuccess && dt == DB_BF16) err = allow_shared<__nv_bfloat16>();
    return err == cudaSuccess ? DB_OK : record_cuda_error(err, "db_adamw_plan_create");
}

}  // namespace
}  // namespace dynbatch

struct db_adamw_plan {
    dynbatch::Layout layout{};
    char* table = nullptr;
    db_dtype grad_dtype = DB_F32, state_dtype = DB_F32;
    int32_t K = 0;
    bool clip = false;
    std::mutex launches;         // held while a call enqueues, so that no other thread's kernels come between its own
};

struct db_grad_norm_plan {
    dynbatch::Layout layout{};
    char* table = nullptr;
    db_dtype grad_dtype = DB_F32;
    int32_t K = 0;
    std::mutex launches;
};

namespace dynbatch {
namespace {

bool known(db_dtype dt) { return dt == DB_F32 || dt == DB_BF16; }

// Checks of the gradient table shared by both plans; fills one tensor's part of `read` and tells whether all
// its gradients reach the alignment of a lane's vector (32 bytes fp32, 16 bf16).
db_status check_grads(const void* const* grads, db_dtype dt, int32_t K, int32_t T, int32_t t, long long n,
                      std::vector<Range>* read, bool* aligned) {
    const size_t size = grad_bytes(dt);
    *aligned = true;
    for (int32_t k = 0; k < K; ++k) {
        const void* g = grads[static_cast<size_t>(k) * T + t];
        if (n > 0 && !g) return DB_ERR_NULL;
        if (misaligned(g, size)) return DB_ERR_ARG;
        *aligned = *aligned && !misaligned(g, size * kLaneElems);
        add_range(*read, g, n, size);
    }
    return DB_OK;
}

// Norm records of one tensor; returns the place of the next.
long long* norm_records(long long* r, const Records& kind, const void* const* grads, db_dtype dt, int32_t K, int32_t T,
                        int32_t t, long long n, long long position, bool aligned) {
    for (long long e = 0; e < n; e += kind.run, r += kind.stride) {
        r[kNormCount] = std::min<long long>(n - e, kind.run) | static_cast<long long>(aligned ? kGradsAligned : 0) << 32;
        r[kNormPosition] = position + e;
        for (int32_t k = 0; k < K; ++k)
            r[kNormGrads + k] = word(static_cast<const char*>(grads[static_cast<size_t>(k) * T + t]) + e * grad_bytes(dt));
    }
    return r;
}

}  // namespace
}  // namespace dynbatch

extern "C" size_t db_adamw_plan_device_bytes(int32_t K, db_dtype grad_dtype, db_dtype state_dtype, const int64_t* sizes,
                                             int32_t T, uint32_t flags) {
    using namespace dynbatch;
    if (!sizes || K < 1 || K > DB_MAX_K || T < 1 || !known(grad_dtype) || (flags & ~DB_ADAMW_CLIP)) return 0;
    if (state_dtype != DB_F32 && state_dtype != DB_E4M3) return 0;
    Layout L;
    return make_layout(K, grad_dtype, state_dtype == DB_E4M3, sizes, T, true, flags & DB_ADAMW_CLIP, &L) ? L.end : 0;
}

extern "C" db_status db_adamw_plan_create(db_adamw_plan** out, const void* const* grads, db_dtype grad_dtype,
                                          int32_t K, const int64_t* sizes, int32_t T, float* const* params,
                                          void* const* params_bf16, void* const* first_moment,
                                          void* const* second_moment, db_dtype state_dtype,
                                          float* const* first_scale, float* const* second_scale,
                                          const float* weight_decay, uint32_t flags, void* device_table,
                                          size_t device_table_bytes, void* cuda_stream) {
    using namespace dynbatch;
    if (!out) return DB_ERR_NULL;
    *out = nullptr;
    if (!grads || !sizes || !params || !first_moment || !second_moment || !device_table) return DB_ERR_NULL;
    if (K < 1 || K > DB_MAX_K || T < 1 || (flags & ~DB_ADAMW_CLIP)) return DB_ERR_ARG;
    if (!known(grad_dtype) || (state_dtype != DB_F32 && state_dtype != DB_E4M3)) return DB_ERR_UNSUPPORTED;
    const bool state8 = state_dtype == DB_E4M3, clip = flags & DB_ADAMW_CLIP;
    if (state8 && (!first_scale || !second_scale)) return DB_ERR_NULL;
    try {
        Layout L;
        if (!make_layout(K, grad_dtype, state8, sizes, T, true, clip, &L)) return DB_ERR_ARG;
        if (misaligned(device_table, 256) || device_table_bytes < L.end) return DB_ERR_ARG;
        const size_t state_size = state8 ? 1 : 4;
        std::vector<Range> written, read;
        std::vector<long long> step(static_cast<size_t>(L.step.stride) * static_cast<size_t>(L.step.count), 0);
        std::vector<long long> norm(static_cast<size_t>(L.norm.stride) * static_cast<size_t>(L.norm.count), 0);
        add_range(written, device_table, static_cast<long long>(L.end), 1);
        long long *r = step.data(), *q = norm.data();
        long long position = 0;
        for (int32_t t = 0; t < T; ++t) {
            const long long n = sizes[t], blocks = blocks_of(n);
            const float wd = weight_decay ? weight_decay[t] : 0.0f;
            if (!std::isfinite(wd)) return DB_ERR_ARG;
            float* p = params[t];
            char *m = static_cast<char*>(first_moment[t]), *u = static_cast<char*>(second_moment[t]);
            char* w = params_bf16 ? static_cast<char*>(params_bf16[t]) : nullptr;
            float *ms = state8 ? first_scale[t] : nullptr, *us = state8 ? second_scale[t] : nullptr;
            if (n > 0 && (!p || !m || !u || (params_bf16 && !w) || (state8 && (!ms || !us)))) return DB_ERR_NULL;
            if (misaligned(p, 4) || misaligned(m, state_size) || misaligned(u, state_size) || misaligned(w, 2) ||
                misaligned(ms, 4) || misaligned(us, 4))
                return DB_ERR_ARG;
            add_range(written, p, n, 4);
            add_range(written, m, n, state_size);
            add_range(written, u, n, state_size);
            add_range(written, w, n, 2);
            add_range(written, ms, blocks, 4);
            add_range(written, us, blocks, 4);
            bool grads_aligned;
            const db_status st = check_grads(grads, grad_dtype, K, T, t, n, &read, &grads_aligned);
            if (st != DB_OK) return st;
            // a lane's vector: 32 bytes of fp32; 8-bit moments are copied 16 bytes at a time
            const size_t state_vec = state8 ? 16 : 32;
            const bool state_aligned = !misaligned(p, 32) && !misaligned(m, state_vec) && !misaligned(u, state_vec) &&
                                       !misaligned(w, 16);
            const long long bits = (state_aligned ? kStateAligned : 0) | (grads_aligned ? kGradsAligned : 0);
            uint32_t wd_bits;
            static_assert(sizeof wd_bits == sizeof wd, "binary32");
            __builtin_memcpy(&wd_bits, &wd, 4);
            for (long long e = 0; e < n; e += L.step.run, r += L.step.stride) {
                r[kRecParam] = word(p + e);
                r[kRecFirst] = word(m + e * state_size);
                r[kRecSecond] = word(u + e * state_size);
                r[kRecCount] = std::min<long long>(n - e, L.step.run) | bits << 32;
                if (state8) {
                    r[kRecFirstScale] = word(ms + e / kWarpElems);
                    r[kRecSecondScale] = word(us + e / kWarpElems);
                }
                r[kRecCopy] = w ? word(w + 2 * e) : 0;
                r[kRecDecay] = wd_bits;
                r[kRecPosition] = position + e;
                for (int32_t k = 0; k < K; ++k)
                    r[kRecGrads + k] = word(static_cast<const char*>(grads[static_cast<size_t>(k) * T + t]) + e * grad_bytes(grad_dtype));
            }
            if (clip) q = norm_records(q, L.norm, grads, grad_dtype, K, T, t, n, position, grads_aligned);
            position += blocks * kWarpElems;
        }
        if (overlaps(written, read)) return DB_ERR_ARG;
        db_adamw_plan* plan = new db_adamw_plan();
        plan->layout = L;
        plan->table = static_cast<char*>(device_table);
        plan->grad_dtype = grad_dtype;
        plan->state_dtype = state_dtype;
        plan->K = K;
        plan->clip = clip;
        db_status st = upload(L, step, norm, plan->table, static_cast<cudaStream_t>(cuda_stream), "db_adamw_plan_create");
        if (st == DB_OK && state8) st = allow_shared(grad_dtype);
        if (st != DB_OK) {
            delete plan;
            return st;
        }
        *out = plan;
        return DB_OK;
    } catch (const std::exception&) {
        record_message("db_adamw_plan_create: out of host memory");
        return DB_ERR_UNSUPPORTED;
    }
}

extern "C" db_status db_adamw_plan_destroy(db_adamw_plan* plan) {
    delete plan;
    return DB_OK;
}

extern "C" db_status db_aggregate_adamw_multi(db_adamw_plan* plan, const int32_t* b, float lr, float beta1, float beta2,
                                              float eps, int64_t step, float max_norm, uint64_t seed, float* grad_norm,
                                              void* cuda_stream) {
    using namespace dynbatch;
    if (!plan || !b) return DB_ERR_NULL;
    if (!std::isfinite(lr) || !std::isfinite(eps) || !(eps >= 0.0f) || step < 1) return DB_ERR_ARG;
    if (!(beta1 >= 0.0f) || !(beta1 < 1.0f) || !(beta2 >= 0.0f) || !(beta2 < 1.0f)) return DB_ERR_ARG;
    if (!std::isfinite(max_norm) || !(max_norm >= 0.0f) || (max_norm > 0.0f && !plan->clip)) return DB_ERR_ARG;
    if (misaligned(grad_norm, 4)) return DB_ERR_ARG;
    StepArgs a{};
    const db_status st = set_workers(b, plan->K, &a.src);
    if (st != DB_OK) return st;
    const Layout& L = plan->layout;
    if (L.step.count == 0) return DB_OK;
    const bool clip = max_norm > 0.0f, norm = !clip && grad_norm, staged = clip && stages(a.src.K, plan->grad_dtype);
    a.src.recs = reinterpret_cast<const long long*>(plan->table + L.step.at);
    a.src.records = L.step.count;
    a.src.stride = L.step.stride;
    a.src.staged = staged ? reinterpret_cast<float*>(plan->table + L.staged) : nullptr;
    a.partials = reinterpret_cast<double*>(plan->table + L.partials);
    float* factor = reinterpret_cast<float*>(plan->table + L.scalars) + 1;
    a.factor = factor;
    a.beta1 = pair_of(beta1);
    a.beta2 = pair_of(beta2);
    a.one_minus_beta1 = pair_of(1.0f - beta1);
    a.one_minus_beta2 = pair_of(1.0f - beta2);
    // bias corrections in fp64, once per call
    const double c1 = 1.0 - std::pow(static_cast<double>(beta1), static_cast<double>(step));
    const double c2 = 1.0 - std::pow(static_cast<double>(beta2), static_cast<double>(step));
    a.minus_step_size = pair_of(static_cast<float>(-static_cast<double>(lr) / c1));
    a.inv_sqrt_c2 = pair_of(static_cast<float>(1.0 / std::sqrt(c2)));
    a.eps = pair_of(eps > 0.0f ? std::max(eps, 1.17549435e-38f) : 0.0f);      // never subnormal: see the kernel's reciprocal
    a.lr = lr;
    // keys of the stochastic rounding: the finalizer of splitmix64 (Steele, Lea and Flood 2014) over seed and step
    uint64_t z = seed + 0x9E3779B97F4A7C15ull * static_cast<uint64_t>(step);
    z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ z >> 27) * 0x94D049BB133111EBull;
    z ^= z >> 31;
    a.key0 = static_cast<uint32_t>(z);
    a.key1 = static_cast<uint32_t>(z >> 32);

    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const std::lock_guard<std::mutex> together(plan->launches);
    if (clip) {
        a.norm = grad_norm;
        a.max_norm = max_norm;
        const db_status s = launch_norm(L, plan->table, plan->grad_dtype, plan->K, a.src, grad_norm, factor, max_norm,
                                        &a.partial_count, stream);
        if (s != DB_OK) return s;
    }
    const int K = staged ? 1 : a.src.K;
    StepFn fn;
    size_t shared = 0;
    if (plan->state_dtype == DB_E4M3) {
        // a staged aggregate is one fp32 gradient, whatever the workers' are
        fn = plan->grad_dtype == DB_F32 || staged ? pick_step8<float>(K, clip, norm, &shared)
                                                  : pick_step8<__nv_bfloat16>(K, clip, norm, &shared);
    } else {
        fn = plan->grad_dtype == DB_F32 ? pick_step<float>(K, clip, norm) : pick_step<__nv_bfloat16>(K, clip, norm);
    }
    DB_CUDA_TRY(launch(fn, L.step.count, kThreads, shared, stream, a));
    return norm ? launch_fold(L, plan->table, L.step.count, grad_norm, nullptr, 0.0f, stream) : DB_OK;
}

extern "C" size_t db_grad_norm_plan_device_bytes(int32_t K, db_dtype grad_dtype, const int64_t* sizes, int32_t T) {
    using namespace dynbatch;
    if (!sizes || K < 1 || K > DB_MAX_K || T < 1 || !known(grad_dtype)) return 0;
    Layout L;
    return make_layout(K, grad_dtype, false, sizes, T, false, true, &L) ? L.end : 0;
}

extern "C" db_status db_grad_norm_plan_create(db_grad_norm_plan** out, const void* const* grads, db_dtype grad_dtype,
                                              int32_t K, const int64_t* sizes, int32_t T, void* device_table,
                                              size_t device_table_bytes, void* cuda_stream) {
    using namespace dynbatch;
    if (!out) return DB_ERR_NULL;
    *out = nullptr;
    if (!grads || !sizes || !device_table) return DB_ERR_NULL;
    if (K < 1 || K > DB_MAX_K || T < 1) return DB_ERR_ARG;
    if (!known(grad_dtype)) return DB_ERR_UNSUPPORTED;
    try {
        Layout L;
        if (!make_layout(K, grad_dtype, false, sizes, T, false, true, &L)) return DB_ERR_ARG;
        if (misaligned(device_table, 256) || device_table_bytes < L.end) return DB_ERR_ARG;
        std::vector<Range> written, read;
        std::vector<long long> norm(static_cast<size_t>(L.norm.stride) * static_cast<size_t>(L.norm.count), 0);
        add_range(written, device_table, static_cast<long long>(L.end), 1);
        long long *r = norm.data(), position = 0;
        for (int32_t t = 0; t < T; ++t) {
            const long long n = sizes[t];
            bool aligned;
            const db_status st = check_grads(grads, grad_dtype, K, T, t, n, &read, &aligned);
            if (st != DB_OK) return st;
            r = norm_records(r, L.norm, grads, grad_dtype, K, T, t, n, position, aligned);
            position += blocks_of(n) * kWarpElems;
        }
        if (overlaps(written, read)) return DB_ERR_ARG;
        db_grad_norm_plan* plan = new db_grad_norm_plan();
        plan->layout = L;
        plan->table = static_cast<char*>(device_table);
        plan->grad_dtype = grad_dtype;
        plan->K = K;
        const db_status st = upload(L, {}, norm, plan->table, static_cast<cudaStream_t>(cuda_stream), "db_grad_norm_plan_create");
        if (st != DB_OK) {
            delete plan;
            return st;
        }
        *out = plan;
        return DB_OK;
    } catch (const std::exception&) {
        record_message("db_grad_norm_plan_create: out of host memory");
        return DB_ERR_UNSUPPORTED;
    }
}

extern "C" db_status db_grad_norm_plan_destroy(db_grad_norm_plan* plan) {
    delete plan;
    return DB_OK;
}

extern "C" db_status db_grad_norm_multi(db_grad_norm_plan* plan, const int32_t* b, float* grad_norm, void* cuda_stream) {
    using namespace dynbatch;
    if (!plan || !b || !grad_norm) return DB_ERR_NULL;
    if (misaligned(grad_norm, 4)) return DB_ERR_ARG;
    Source src{};
    const db_status st = set_workers(b, plan->K, &src);
    if (st != DB_OK) return st;
    if (plan->layout.norm.count == 0) return DB_OK;
    const std::lock_guard<std::mutex> together(plan->launches);
    return launch_norm(plan->layout, plan->table, plan->grad_dtype, plan->K, src, grad_norm, nullptr, 0.0f, nullptr,
                       static_cast<cudaStream_t>(cuda_stream));
}
