// Host side of the training operators (include/egeria_ops.h): argument checks, plans, launches.
#include <cmath>
#include <new>
#include <vector>

#include "adamw.cuh"
#include "norm.cuh"
#include "ops_host.h"

namespace egeria {
namespace ops {

struct LinearLayout {
    size_t part, part2, x, w, dz, sums, total;
};
static LinearLayout linear_layout(int64_t rows, int64_t inp, int64_t out) {
    LinearLayout L;
    size_t off = kHeadBytes;
    auto take = [&](size_t n) {
        const size_t at = off;
        off = up(off + n, 1024);
        return at;
    };
    L.part = take(std::max(split_bytes(rows, out, inp), split_bytes(out, inp, rows)));  // z, or dw
    L.part2 = take(split_bytes(rows, inp, out));                                        // dx, in one launch with dw
    L.x = take((size_t)rows * pad8(inp) * 2);
    L.w = take((size_t)out * pad8(inp) * 2);
    L.dz = take((size_t)rows * pad8(out) * 2);
    L.sums = take((size_t)slope_sums(rows, out) * 4);
    L.total = off;
    return L;
}

// ---------------------------------------------------------------- norms
struct NormPlan {
    int team, ctas;  // threads, and thread blocks, of the backward pass
};
static NormPlan norm_backward_plan(int64_t rows, int64_t cols) {
    NormPlan n{32, 16};
    if (cols > 4096) n = {1024, 1};
    else if (cols > 2048) n = {512, 1};
    else if (cols > 1024) n = {256, 2};
    else if (cols > 512) n = {128, 4};
    else if (cols > 256) n = {64, 8};
    n.ctas = (int)std::max<int64_t>(std::min<int64_t>(rows, 1), std::min<int64_t>(rows / 2, (int64_t)n.ctas * kSms));
    return n;
}
// CTAs times columns at most, for these sizes and all smaller ones: 4096 columns' worth per SM (less of it between the
// teams' widths), beyond that one CTA per SM.
static int64_t norm_sums_cols(int64_t rows, int64_t cols) {
    return std::min(std::max<int64_t>(std::min<int64_t>(rows, 1), rows / 2) * cols, kSms * std::max<int64_t>(4096, cols));
}

}  // namespace ops
}  // namespace egeria

using namespace egeria;
using namespace egeria::ops;

namespace egeria {
namespace ops {

template <typename T, int ROWS>
static cudaError_t allow_few() {
    cudaError_t e = cudaFuncSetAttribute(linear_few_kernel<T, ROWS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(linear_few_kernel<T, ROWS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    return e;
}
template <typename T>
static cudaError_t allow_all() {
    cudaError_t e = allow_smem<T, 64, 1, 1, kModeLinear>();
    if (e == cudaSuccess) e = allow_smem<T, 128, 1, 1, kModeLinear>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 1, 1, kModeLinear>();
    if (e == cudaSuccess) e = allow_smem<T, 128, 2, 1, kModeLinear>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 2, 1, kModeLinear>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 2, 2, kModeLinear>();
    if (e == cudaSuccess) e = allow_few<T, 1>();
    if (e == cudaSuccess) e = allow_few<T, 2>();
    if (e == cudaSuccess) e = allow_few<T, 4>();
    return e;
}

template <typename T>
static cudaError_t launch_gemm_any(int bn, int cg, int mb, const GemmParams<kModeLinear> &p, int ctas, cudaStream_t stream) {
    if (mb == 2) return launch_gemm<T, 256, 2, 2, kModeLinear>(p, ctas, stream);
    if (cg == 2) return bn == 128 ? launch_gemm<T, 128, 2, 1, kModeLinear>(p, ctas, stream) : launch_gemm<T, 256, 2, 1, kModeLinear>(p, ctas, stream);
    if (bn == 64) return launch_gemm<T, 64, 1, 1, kModeLinear>(p, ctas, stream);
    return bn == 128 ? launch_gemm<T, 128, 1, 1, kModeLinear>(p, ctas, stream) : launch_gemm<T, 256, 1, 1, kModeLinear>(p, ctas, stream);
}

egeria_status run_products(egeria_ops *o, cudaStream_t stream, int type, Product *jobs, int count, const ColumnSums &sums) {
    // the tile that suits the launch: of the plans of each product, the one that is best for all of them
    GemmPlan plan[2];
    double best = 1e300;
    for (int i = 0; i < count; ++i) {
        const GemmPlan lead = plan_gemm(jobs[i].m, jobs[i].n, jobs[i].k, o->sms);
        GemmPlan g[2];
        double t = 0.0;
        for (int j = 0; j < count; ++j) {
            g[j] = j == i ? lead : plan_tile(jobs[j].m, jobs[j].n, jobs[j].k, o->sms, lead.bn, lead.cg);
            t += gemm_cycles(g[j], (jobs[j].k + kGemmK - 1) / kGemmK, o->sms);
        }
        if (t < best) {
            best = t;
            for (int j = 0; j < count; ++j) plan[j] = g[j];
        }
    }
    // Tiles of 512 rows take a quarter less from L2, but nothing hides their epilogue: for long sums with a light one, where they
    // need no more rounds.  16384 x 2816 -> 1024 with a residual 85 us instead of 92, 8192 x 8192 -> 8192 752 instead of 949; but
    // 8192 x 2048 -> 2048 93 instead of 86, 16384 x 1024 -> 4096 with activation and z 191 instead of 159.  Over sums of 2560 to 8192, 512 to
    // 4096 columns and 2048 to 32768 rows (96 sizes, both in turn) it gains 0 to 7 % at 2560 and 13 to 15 % at 8192 wherever it is taken; the
    // one size that came out slower, 4096 x 2560 -> 4096, did by 2 % with 12 % between its runs.
    if (count == 1 && plan[0].cg == 2 && plan[0].bn == 256 && plan[0].splits == 1 && jobs[0].k >= 40 * kGemmK && !jobs[0].epi.act && !jobs[0].epi.z &&
        !jobs[0].epi.slope) {
        const int64_t workers = o->sms / 2, tall = (jobs[0].m + 511) / 512;
        auto rounds = [&](int64_t tiles) { return (tiles + workers - 1) / workers; };
        if (2 * rounds(tall * plan[0].tiles_n) <= rounds((int64_t)plan[0].tiles_m * plan[0].tiles_n)) plan[0].mb = 2, plan[0].tiles_m = (int)tall;
    }
    GemmParams<kModeLinear> p;
    int ctas = 0;
    const egeria_status s = fill_products(o, type, jobs, plan, count, p, ctas);
    if (s != EGERIA_OK) return s;
    p.sums[0] = sums;
    const int bn = plan[0].bn, cg = plan[0].cg, mb = plan[0].mb;
    EGO_CUDA(type == EGERIA_BF16 ? launch_gemm_any<bf16>(bn, cg, mb, p, ctas, stream) : launch_gemm_any<f16>(bn, cg, mb, p, ctas, stream));
    ++o->launches;
    return EGERIA_OK;
}

egeria_status run_prepare(egeria_ops *o, cudaStream_t stream, int type, const PrepareParams &p, bool wide) {
    int64_t blocks = (int64_t)p.slope.strips * p.slope.runs;
    for (const PackJob &j : p.pack) blocks += j.blocks;
    if (blocks == 0) return EGERIA_OK;
    if (blocks > 0x7fffffff) return EGERIA_ERR_UNSUPPORTED_SHAPE;
    auto go = [&](auto kernel) { return launch(kernel, dim3((unsigned)blocks), 32 * kPrepareWarps, 0, stream, 1, p); };
    EGO_CUDA(type == EGERIA_BF16 ? (wide ? go(prepare_kernel<bf16, true>) : go(prepare_kernel<bf16, false>))
                                 : (wide ? go(prepare_kernel<f16, true>) : go(prepare_kernel<f16, false>)));
    ++o->launches;
    return EGERIA_OK;
}

template <typename T, int ROWS>
static cudaError_t launch_few(const Epilogue &e, const egeria_linear_forward_args &a, bool wide, int sms, cudaStream_t stream) {
    const int smem = ROWS * (int)((a.inp + 255) / 256 * 256) * 2;
    const int grid = (int)std::min<int64_t>((a.out + 7) / 8, (int64_t)sms * 4);
    const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.w);
    return launch(wide ? linear_few_kernel<T, ROWS, true> : linear_few_kernel<T, ROWS, false>, dim3(grid), 256, smem, stream, 1, e,
                  (int32_t)a.rows, (int32_t)a.out, x, a.ldx, w, a.ldw, (int32_t)a.inp);
}
template <typename T>
static cudaError_t launch_few_any(const Epilogue &e, const egeria_linear_forward_args &a, bool wide, int sms, cudaStream_t stream) {
    if (a.rows <= 1) return launch_few<T, 1>(e, a, wide, sms, stream);
    if (a.rows <= 2) return launch_few<T, 2>(e, a, wide, sms, stream);
    return launch_few<T, 4>(e, a, wide, sms, stream);
}

// ---------------------------------------------------------------- norm launches
template <typename T, int TEAM, int VPT>
static cudaError_t norm_fwd(const NormParams &p, bool wide, cudaStream_t stream) {
    const int64_t per = TEAM == 32 ? 4 : 1;
    const unsigned grid = (unsigned)((p.rows + per - 1) / per);
    const int threads = TEAM == 32 ? 128 : TEAM;
    auto go = [&](auto kernel) { return launch(kernel, dim3(grid), threads, 0, stream, 1, p); };
    if (wide && p.cols == TEAM * VPT * 8) return go(norm_forward_kernel<T, TEAM, VPT, true, true>);
    return wide ? go(norm_forward_kernel<T, TEAM, VPT, true, false>) : go(norm_forward_kernel<T, TEAM, VPT, false, false>);
}
template <typename T>
static cudaError_t norm_fwd_any(const NormParams &p, bool wide, cudaStream_t stream) {
    if (p.cols <= 256) return norm_fwd<T, 32, 1>(p, wide, stream);
    if (p.cols <= 512) return norm_fwd<T, 32, 2>(p, wide, stream);
    if (p.cols <= 768) return norm_fwd<T, 32, 3>(p, wide, stream);
    if (p.cols <= 1024) return norm_fwd<T, 32, 4>(p, wide, stream);
    if (p.cols <= 4096) return norm_fwd<T, 128, 4>(p, wide, stream);
    return norm_fwd<T, 256, 4>(p, wide, stream);
}
template <typename T, int TEAM>
static cudaError_t norm_bwd(const NormParams &p, int ctas, bool wide, bool layer, cudaStream_t stream) {
    const size_t smem = wide ? (size_t)norm_ring_rows<T, TEAM>() * 4 * TEAM * sizeof(Raw8<T>) : 0;
    auto go = [&](auto kernel) {
        if (smem > 40 * 1024) {  // with the static part: beyond what needs no permission
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
        }
        return launch(kernel, dim3(ctas), TEAM, smem, stream, 1, p);
    };
    if (wide && p.cols == TEAM * 8) return layer ? go(norm_backward_kernel<T, TEAM, true, true, true>) : go(norm_backward_kernel<T, TEAM, true, true, false>);
    if (wide) return layer ? go(norm_backward_kernel<T, TEAM, true, false, true>) : go(norm_backward_kernel<T, TEAM, true, false, false>);
    return layer ? go(norm_backward_kernel<T, TEAM, false, false, true>) : go(norm_backward_kernel<T, TEAM, false, false, false>);
}
template <typename T>
static cudaError_t norm_bwd_any(const NormParams &p, const NormPlan &n, bool wide, bool layer, bool sums, cudaStream_t stream) {
    cudaError_t e;
    switch (n.team) {
        case 32: e = norm_bwd<T, 32>(p, n.ctas, wide, layer, stream); break;
        case 64: e = norm_bwd<T, 64>(p, n.ctas, wide, layer, stream); break;
        case 128: e = norm_bwd<T, 128>(p, n.ctas, wide, layer, stream); break;
        case 256: e = norm_bwd<T, 256>(p, n.ctas, wide, layer, stream); break;
        case 512: e = norm_bwd<T, 512>(p, n.ctas, wide, layer, stream); break;
        default: e = norm_bwd<T, 1024>(p, n.ctas, wide, layer, stream); break;
    }
    if (e != cudaSuccess || !sums) return e;
    const unsigned strips = (unsigned)((p.cols + 31) / 32);
    const bool long_groups = p.gate_rows > kLongGroup * p.cta_rows;  // then there are at most CTAs / kLongGroup + 1 groups
    unsigned gates = 0;
    if (p.dgate) gates = (unsigned)(long_groups ? (p.rows + p.gate_rows - 1) / p.gate_rows : (n.ctas - 1 + 31) / 32);
    return launch(norm_sums_kernel<T>, dim3(strips, 4 + gates), kSumsThreads, 0, stream, 1, p, n.ctas, (int)long_groups);
}

static egeria_status device_ready(int *sms) {
    int dev = 0, major = 0;
    EGO_CUDA(cudaGetDevice(&dev));
    EGO_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    if (major != 10) return EGERIA_ERR_UNSUPPORTED_DEVICE;
    EGO_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    return EGERIA_OK;
}

// ---------------------------------------------------------------- AdamW tables
typedef void (*AdamKernel)(AdamParams);
template <bool SMALL>
static AdamKernel adam_kernel(int p, int g, bool master) {
    if (p == EGERIA_F32) return master ? adamw_kernel<float, float, true, SMALL> : adamw_kernel<float, float, false, SMALL>;
    if (p == EGERIA_BF16) {
        if (g == EGERIA_F32) return master ? adamw_kernel<bf16, float, true, SMALL> : adamw_kernel<bf16, float, false, SMALL>;
        return master ? adamw_kernel<bf16, bf16, true, SMALL> : adamw_kernel<bf16, bf16, false, SMALL>;
    }
    if (g == EGERIA_F32) return master ? adamw_kernel<f16, float, true, SMALL> : adamw_kernel<f16, float, false, SMALL>;
    return master ? adamw_kernel<f16, f16, true, SMALL> : adamw_kernel<f16, f16, false, SMALL>;
}
// Tensors of one combination of types go through one launch.
constexpr int kAdamClasses = 18;
static int adam_class(const egeria_adamw_tensor &t) { return (t.param_type * 3 + t.grad_type) * 2 + (t.master ? 1 : 0); }

static bool good_adam_tensor(const egeria_adamw_tensor &t, uint32_t flags) {
    if (t.n < 0 || t.param_type < EGERIA_F32 || t.param_type > EGERIA_F16 || t.module < -1) return false;
    if (t.grad_type != EGERIA_F32 && t.grad_type != t.param_type) return false;
    if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay)) return false;
    if (t.n == 0) return true;
    if (!t.param || !t.m || !t.v || !aligned(t.param, size_of(t.param_type)) || !aligned(t.master, 4)) return false;
    if (flags & EGERIA_ADAMW_8BIT) return t.m_scale && t.v_scale && aligned(t.m_scale, 4) && aligned(t.v_scale, 4);
    return aligned(t.m, 4) && aligned(t.v, 4);
}

struct AdamLayout {
    size_t tensors, grads, chunks, tickets, total;
    int64_t n_chunks;
};
static bool adam_layout(int count, const egeria_adamw_tensor *t, AdamLayout &L) {
    L.n_chunks = 0;
    for (int i = 0; i < count; ++i) {
        const int64_t c = (t[i].n + kAdamChunk - 1) / kAdamChunk;
        if (t[i].n < 0 || c > 0x7fffffff) return false;
        L.n_chunks += c;
    }
    if (L.n_chunks > 0x7fffffff) return false;
    L.tickets = 0;  // [0] status words, then one ticket per class, 128 bytes apart
    L.tensors = 128 * (1 + kAdamClasses);
    L.grads = up(L.tensors + (size_t)count * sizeof(AdamTensor), kAlign);
    L.chunks = up(L.grads + (size_t)count * sizeof(void *), kAlign);
    L.total = up(L.chunks + (size_t)L.n_chunks * sizeof(int2), kAlign);
    return true;
}

// Whether a forward call goes without the tensor cores, and needs no workspace.
static bool linear_few(const egeria_linear_forward_args &a) {
    const int few_rows = a.rows <= 2 ? (int)a.rows : 4;
    return a.rows <= kFewRows && (a.inp + 255) / 256 * 256 * 2 * few_rows <= kFewSmem;
}
egeria_status linear_forward_at(egeria_ops *ops, cudaStream_t stream, const egeria_linear_forward_args &a, size_t part, size_t x, size_t w) {
    Epilogue e{};
    e.bias = a.bias;
    e.extra = a.residual;
    e.ldx = a.ldr;
    e.out = a.y;
    e.ldo = a.ldy;
    e.z = a.z;
    e.ldz = a.ldz;
    e.act = a.act;
    if (linear_few(a)) {
        const bool wide = a.inp % 8 == 0 && a.ldw % 8 == 0 && aligned(a.w, 16);
        EGO_CUDA(a.type == EGERIA_BF16 ? launch_few_any<bf16>(e, a, wide, ops->sms, stream) : launch_few_any<f16>(e, a, wide, ops->sms, stream));
        ++ops->launches;
        return EGERIA_OK;
    }
    PrepareParams prep{};
    prep.status = reinterpret_cast<int32_t *>(ops->ws);
    Product job{a.rows, a.out, a.inp, {a.x, a.ldx, a.rows, a.inp, false}, {a.w, a.ldw, a.out, a.inp, false}, {e}, part};
    make_loadable(ops, job.a, x, prep.pack[0]);
    make_loadable(ops, job.b, w, prep.pack[1]);
    const egeria_status s = run_prepare(ops, stream, a.type, prep, false);
    return s != EGERIA_OK ? s : run_products(ops, stream, a.type, &job, 1, ColumnSums{});
}

}  // namespace ops
}  // namespace egeria

struct egeria_adamw {
    struct Class {
        AdamKernel kernel;
        AdamParams params;
        int grid;
    };
    std::vector<Class> classes;
    uint8_t *ws = nullptr;
    AdamLayout L{};
    int count = 0;
    std::vector<size_t> grad_size;   // 0 for an empty tensor
    int64_t launches = 0;
    cudaStream_t last_stream = nullptr;
};

extern "C" {

// ---------------------------------------------------------------- handle
egeria_status egeria_ops_create(egeria_ops **out, void *workspace, size_t workspace_bytes) {
    if (!out) return EGERIA_ERR_INVALID_ARG;
    *out = nullptr;
    if (!workspace || !aligned(workspace, EGERIA_WORKSPACE_ALIGN) || workspace_bytes < EGERIA_OPS_WORKSPACE_MIN) return EGERIA_ERR_WORKSPACE;
    int sms = 0;
    egeria_status s = device_ready(&sms);
    if (s != EGERIA_OK) return s;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) {
        (void)cudaGetLastError();
        return EGERIA_ERR_CUDA;
    }
    EGO_CUDA(allow_all<bf16>());
    EGO_CUDA(allow_all<f16>());
    // the workspace may be memory that earlier work of a stream which the default stream does not wait for still writes to
    EGO_CUDA(cudaDeviceSynchronize());
    EGO_CUDA(cudaMemset(workspace, 0, kHeadBytes));
    EGO_CUDA(cudaDeviceSynchronize());
    egeria_ops *o = new (std::nothrow) egeria_ops();
    if (!o) return EGERIA_ERR_INVALID_ARG;
    o->ws = static_cast<uint8_t *>(workspace);
    o->ws_bytes = workspace_bytes;
    o->encode = reinterpret_cast<EncodeTiledFn>(fn);
    o->sms = std::min(sms, kMaxSplitCtas);
    *out = o;
    return EGERIA_OK;
}
egeria_status egeria_ops_destroy(egeria_ops *ops) {
    if (!ops) return EGERIA_ERR_INVALID_ARG;
    delete ops;
    return EGERIA_OK;
}
egeria_status egeria_ops_device_status(egeria_ops *ops) {
    if (!ops) return EGERIA_ERR_INVALID_ARG;
    EGO_CUDA(cudaStreamSynchronize(ops->last_stream));
    int32_t v = 0;
    EGO_CUDA(cudaMemcpy(&v, ops->ws, sizeof(v), cudaMemcpyDeviceToHost));
    if (v == 0) return EGERIA_OK;
    // tickets too: a call that gave up may have left some.  In the call's own stream, which need not wait for the default one
    EGO_CUDA(cudaMemsetAsync(ops->ws, 0, kHeadBytes, ops->last_stream));
    EGO_CUDA(cudaStreamSynchronize(ops->last_stream));
    return static_cast<egeria_status>(v);
}
int64_t egeria_ops_launch_count(const egeria_ops *ops) { return ops ? ops->launches : 0; }
egeria_status egeria_ops_debug_stall_next(egeria_ops *ops, int kind) {
    if (!ops || kind < 0 || kind > 2) return EGERIA_ERR_INVALID_ARG;
    ops->stall_next = (uint32_t)kind;
    return EGERIA_OK;
}

// ---------------------------------------------------------------- linear
size_t egeria_linear_workspace_bytes(int64_t rows, int64_t inp, int64_t out) {
    if (good_sizes(rows, inp, out) != EGERIA_OK) return 0;
    return linear_layout(rows, inp, out).total;
}

egeria_status egeria_linear_forward(egeria_ops *ops, void *cuda_stream, const egeria_linear_forward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_linear_forward_args &a = *args;
    if ((a.type != EGERIA_BF16 && a.type != EGERIA_F16) || !good_act(a.act)) return EGERIA_ERR_INVALID_ARG;
    egeria_status s = good_sizes(a.rows, a.inp, a.out);
    if (s != EGERIA_OK) return s;
    if (a.rows == 0) return EGERIA_OK;
    if (!good_matrix(a.x, a.ldx, a.inp, 2) || !good_matrix(a.w, a.ldw, a.inp, 2) || !good_matrix(a.y, a.ldy, a.out, 2) ||
        !good_optional(a.residual, a.ldr, a.out, 2) || !good_optional(a.z, a.ldz, a.out, 2) || !aligned(a.bias, 2))
        return EGERIA_ERR_INVALID_ARG;
    // blocks write y and z while others still read; a residual is read where the same thread writes y
    const Extent y{a.y, a.ldy, a.rows, a.out}, z{a.z, a.ldz, a.rows, a.out};
    const Extent reads[4] = {{a.x, a.ldx, a.rows, a.inp}, {a.w, a.ldw, a.out, a.inp}, {a.bias, a.out, 1, a.out}, {a.residual, a.ldr, a.rows, a.out}};
    const bool onto = a.residual == a.y && (a.ldr == a.ldy || a.rows == 1);
    for (int i = 0; i < 4; ++i)
        if ((!(i == 3 && onto) && overlap(y, reads[i])) || overlap(z, reads[i])) return EGERIA_ERR_INVALID_ARG;
    if (overlap(y, z)) return EGERIA_ERR_INVALID_ARG;
    const LinearLayout L = linear_layout(a.rows, a.inp, a.out);
    if (!linear_few(a) && ops->ws_bytes < L.total) return EGERIA_ERR_WORKSPACE;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    ops->last_stream = stream;
    return linear_forward_at(ops, stream, a, L.part, L.x, L.w);
}

egeria_status egeria_linear_backward(egeria_ops *ops, void *cuda_stream, const egeria_linear_backward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_linear_backward_args &a = *args;
    if ((a.type != EGERIA_BF16 && a.type != EGERIA_F16) || !good_act(a.act) || !good_act(a.act_in)) return EGERIA_ERR_INVALID_ARG;
    egeria_status s = good_sizes(a.rows, a.inp, a.out);
    if (s != EGERIA_OK) return s;
    if (!good_optional(a.dx, a.lddx, a.inp, 2) || !good_optional(a.dw, a.lddw, a.inp, 2) || !aligned(a.db, 2)) return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (a.rows == 0) {
        ops->last_stream = stream;
        if (a.dw) EGO_CUDA(cudaMemset2DAsync(a.dw, (size_t)a.lddw * 2, 0, (size_t)a.inp * 2, (size_t)a.out, stream));
        if (a.db) EGO_CUDA(cudaMemsetAsync(a.db, 0, (size_t)a.out * 2, stream));
        return EGERIA_OK;
    }
    if (!good_matrix(a.dy, a.lddy, a.out, 2)) return EGERIA_ERR_INVALID_ARG;
    if (a.act != EGERIA_ACT_NONE && !good_matrix(a.z, a.ldz, a.out, 2)) return EGERIA_ERR_INVALID_ARG;
    if (a.dw && !good_matrix(a.x, a.ldx, a.inp, 2)) return EGERIA_ERR_INVALID_ARG;
    if (a.dx && !good_matrix(a.w, a.ldw, a.inp, 2)) return EGERIA_ERR_INVALID_ARG;
    if (a.dx && a.act_in != EGERIA_ACT_NONE && !good_matrix(a.z_in, a.ldz_in, a.inp, 2)) return EGERIA_ERR_INVALID_ARG;
    const LinearLayout L = linear_layout(a.rows, a.inp, a.out);
    if (ops->ws_bytes < L.total) return EGERIA_ERR_WORKSPACE;
    ops->last_stream = stream;

    const bool products = a.dx || a.dw;
    Operand dz{a.dy, a.lddy, a.rows, a.out, false};
    const bool own_dz = products && (a.act != EGERIA_ACT_NONE || !aligned(a.dy, 16) || a.lddy % 8 != 0);
    if (own_dz) {
        dz.p = ops->ws + L.dz;
        dz.ld = pad8(a.out);
    }
    PrepareParams prep{};
    prep.status = reinterpret_cast<int32_t *>(ops->ws);
    ColumnSums sums{};
    bool wide = false;
    if (own_dz || a.db) {
        SlopeJob &j = prep.slope;
        j.dz = own_dz ? ops->ws + L.dz : nullptr;
        j.lddz = dz.ld;
        j.dy = a.dy;
        j.lddy = a.lddy;
        j.z = a.act == EGERIA_ACT_NONE ? nullptr : a.z;
        j.ldz = a.ldz;
        j.act = a.act;
        j.rows = a.rows;
        j.cols = (int32_t)a.out;
        j.strips = (int32_t)((a.out + 255) / 256);
        j.runs = slope_runs(a.rows, a.out);
        j.db = a.db;
        if (a.db) {
            j.sums = reinterpret_cast<float *>(ops->ws + L.sums);
            j.sums_room = slope_sums(a.rows, a.out);
            if (j.runs > 1) sums = ColumnSums{j.sums, a.db, j.runs, j.cols};
        }
        wide = a.out % 8 == 0 && aligned(a.dy, 16) && a.lddy % 8 == 0 && (!j.z || (aligned(j.z, 16) && a.ldz % 8 == 0));
    }
    Product jobs[2];
    int count = 0;
    if (a.dw) {  // first: its sums are the longer ones as a rule, and dx's tiles fill what it leaves
        Operand dzt = dz;
        dzt.mn = true;
        Product &j = jobs[count++] = Product{a.out, a.inp, a.rows, dzt, {a.x, a.ldx, a.rows, a.inp, true}, {}, L.part};
        j.epi.out = a.dw;
        j.epi.ldo = a.lddw;
        make_loadable(ops, j.b, L.x, prep.pack[0]);
    }
    if (a.dx) {
        Product &j = jobs[count++] = Product{a.rows, a.inp, a.out, dz, {a.w, a.ldw, a.out, a.inp, true}, {}, L.part2};
        j.epi.out = a.dx;
        j.epi.ldo = a.lddx;
        if (a.act_in != EGERIA_ACT_NONE) {
            j.epi.extra = a.z_in;
            j.epi.ldx = a.ldz_in;
            j.epi.act_in = a.act_in;
            j.epi.slope = 1;
        }
        make_loadable(ops, j.b, L.w, prep.pack[1]);
    }
    if ((s = run_prepare(ops, stream, a.type, prep, wide)) != EGERIA_OK) return s;
    if (count) return run_products(ops, stream, a.type, jobs, count, sums);
    if (sums.out) {
        const dim3 grid((unsigned)((a.out + 31) / 32));
        EGO_CUDA(a.type == EGERIA_BF16 ? launch(add_columns_kernel<bf16>, grid, 512, 0, stream, 1, sums)
                                       : launch(add_columns_kernel<f16>, grid, 512, 0, stream, 1, sums));
        ++ops->launches;
    }
    return EGERIA_OK;
}

// ---------------------------------------------------------------- norms
size_t egeria_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || cols > EGERIA_NORM_MAX_COLS) return 0;
    return kHeadBytes + up((size_t)norm_sums_cols(rows, cols) * kNormSums * 4, 1024);
}

egeria_status egeria_norm_forward(egeria_ops *ops, void *cuda_stream, const egeria_norm_forward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_norm_forward_args &a = *args;
    if (a.type < EGERIA_F32 || a.type > EGERIA_F16 || (a.param_type != EGERIA_F32 && a.param_type != a.type) ||
        (a.kind != EGERIA_NORM_LAYER && a.kind != EGERIA_NORM_RMS) || a.rows < 0 || a.cols < 1 || a.gate_rows < 0 || !(a.eps >= 0.0f))
        return EGERIA_ERR_INVALID_ARG;
    if (a.cols > EGERIA_NORM_MAX_COLS || a.rows > kMaxSize) return EGERIA_ERR_UNSUPPORTED_SHAPE;
    if (a.rows == 0) return EGERIA_OK;
    const size_t e = size_of(a.type), pe = size_of(a.param_type);
    if (!good_matrix(a.x, a.ldx, a.cols, e) || !good_matrix(a.f, a.ldf, a.cols, e) || !good_matrix(a.y, a.ldy, a.cols, e) ||
        (a.pre && !good_matrix(a.h, a.ldh, a.cols, e)) || !aligned(a.stats, 16))
        return EGERIA_ERR_INVALID_ARG;
    const void *vec[5] = {a.gate, a.w_post, a.b_post, a.w_pre, a.b_pre};
    const size_t row_align = 8 * e, vec_align = 8 * pe;
    bool wide = a.cols % 8 == 0 && aligned(a.x, row_align) && aligned(a.f, row_align) && aligned(a.y, row_align) && a.ldx % 8 == 0 &&
                a.ldf % 8 == 0 && a.ldy % 8 == 0 && (!a.pre || (aligned(a.h, row_align) && a.ldh % 8 == 0));
    for (const void *v : vec) {
        if (!aligned(v, pe)) return EGERIA_ERR_INVALID_ARG;
        wide = wide && aligned(v, vec_align);
    }
    NormParams p;
    memset(&p, 0, sizeof(p));
    p.x = a.x, p.ldx = a.ldx;
    p.f = a.f, p.ldf = a.ldf;
    p.gate = a.gate;
    if (a.post) p.w_post = a.w_post, p.b_post = a.b_post;
    if (a.pre) p.w_pre = a.w_pre, p.b_pre = a.b_pre;
    p.y = a.y, p.ldy = a.ldy;
    p.h = a.h, p.ldh = a.ldh;
    p.stats = a.stats;
    p.rows = a.rows;
    p.gate_rows = a.gate_rows ? a.gate_rows : a.rows;
    p.cols = (int32_t)a.cols;
    p.layer = a.kind == EGERIA_NORM_LAYER;
    p.post = a.post != 0;
    p.pre = a.pre != 0;
    p.w_float = a.param_type == EGERIA_F32;
    p.alpha = a.alpha;
    p.eps = a.eps;
    p.inv_cols = 1.0f / (float)a.cols;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    ops->last_stream = stream;
    EGO_CUDA(a.type == EGERIA_F32    ? norm_fwd_any<float>(p, wide, stream)
             : a.type == EGERIA_BF16 ? norm_fwd_any<bf16>(p, wide, stream)
                                     : norm_fwd_any<f16>(p, wide, stream));
    ++ops->launches;
    return EGERIA_OK;
}

egeria_status egeria_norm_backward(egeria_ops *ops, void *cuda_stream, const egeria_norm_backward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_norm_backward_args &a = *args;
    if (a.type < EGERIA_F32 || a.type > EGERIA_F16 || (a.param_type != EGERIA_F32 && a.param_type != a.type) ||
        (a.kind != EGERIA_NORM_LAYER && a.kind != EGERIA_NORM_RMS) || a.rows < 0 || a.cols < 1 || a.gate_rows < 0)
        return EGERIA_ERR_INVALID_ARG;
    if (a.cols > EGERIA_NORM_MAX_COLS || a.rows > kMaxSize) return EGERIA_ERR_UNSUPPORTED_SHAPE;
    const size_t e = size_of(a.type), pe = size_of(a.param_type);
    const void *vec[10] = {a.gate, a.w_post, a.b_post, a.w_pre, a.b_pre, a.dgate, a.dw_post, a.db_post, a.dw_pre, a.db_pre};
    for (const void *v : vec)
        if (!aligned(v, pe)) return EGERIA_ERR_INVALID_ARG;
    if ((a.dgate && !a.gate) || (!a.post && (a.dw_post || a.db_post)) || (!a.pre && (a.dw_pre || a.db_pre))) return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (a.rows == 0) {
        ops->last_stream = stream;
        void *const outs[5] = {a.gate_rows == 0 ? a.dgate : nullptr, a.dw_post, a.db_post, a.dw_pre, a.db_pre};
        for (void *o : outs)
            if (o) EGO_CUDA(cudaMemsetAsync(o, 0, (size_t)a.cols * pe, stream));
        return EGERIA_OK;
    }
    if (!good_matrix(a.dy, a.lddy, a.cols, e) || !good_matrix(a.f, a.ldf, a.cols, e) || !good_matrix(a.dx, a.lddx, a.cols, e) ||
        !good_matrix(a.df, a.lddf, a.cols, e) || !a.stats || !aligned(a.stats, 16) ||
        (a.pre && (!good_matrix(a.dh, a.lddh, a.cols, e) || !good_matrix(a.y, a.ldy, a.cols, e))))
        return EGERIA_ERR_INVALID_ARG;
    if (ops->ws_bytes < egeria_norm_workspace_bytes(a.rows, a.cols)) return EGERIA_ERR_WORKSPACE;
    const size_t row_align = 8 * e, vec_align = 8 * pe;
    bool wide = a.cols % 8 == 0 && aligned(a.dy, row_align) && aligned(a.f, row_align) && aligned(a.dx, row_align) && aligned(a.df, row_align) &&
                a.lddy % 8 == 0 && a.ldf % 8 == 0 && a.lddx % 8 == 0 && a.lddf % 8 == 0;
    if (a.pre) wide = wide && aligned(a.dh, row_align) && aligned(a.y, row_align) && a.lddh % 8 == 0 && a.ldy % 8 == 0;
    for (int i = 0; i < 5; ++i) wide = wide && aligned(vec[i], vec_align);
    NormParams p;
    memset(&p, 0, sizeof(p));
    p.x = a.y, p.ldx = a.ldy;
    p.f = a.f, p.ldf = a.ldf;
    p.dy = a.dy, p.lddy = a.lddy;
    p.dh = a.dh, p.lddh = a.lddh;
    p.gate = a.gate;
    if (a.post) p.w_post = a.w_post, p.b_post = a.b_post;
    if (a.pre) p.w_pre = a.w_pre;
    p.y = a.dx, p.ldy = a.lddx;
    p.h = a.df, p.ldh = a.lddf;
    p.stats = const_cast<float *>(a.stats);
    p.sums = reinterpret_cast<float *>(ops->ws + kHeadBytes);
    p.status = reinterpret_cast<int32_t *>(ops->ws);
    p.dw_post = a.dw_post, p.db_post = a.db_post, p.dw_pre = a.dw_pre, p.db_pre = a.db_pre, p.dgate = a.dgate;
    p.rows = a.rows;
    p.gate_rows = a.gate_rows ? a.gate_rows : a.rows;
    p.cols = (int32_t)a.cols;
    p.layer = a.kind == EGERIA_NORM_LAYER;
    p.post = a.post != 0;
    p.pre = a.pre != 0;
    p.w_float = a.param_type == EGERIA_F32;
    p.alpha = a.alpha;
    p.inv_cols = 1.0f / (float)a.cols;
    ops->last_stream = stream;
    const bool layer = p.layer || p.b_post || p.db_pre || p.db_post;  // an rms norm with biases goes with the layer norms
    const NormPlan n = norm_backward_plan(a.rows, a.cols);
    p.cta_rows = a.rows / n.ctas;
    p.extra = a.rows % n.ctas;
    const bool sums = a.dgate || a.dw_post || a.db_post || a.dw_pre || a.db_pre;
    EGO_CUDA(a.type == EGERIA_F32    ? norm_bwd_any<float>(p, n, wide, layer, sums, stream)
             : a.type == EGERIA_BF16 ? norm_bwd_any<bf16>(p, n, wide, layer, sums, stream)
                                     : norm_bwd_any<f16>(p, n, wide, layer, sums, stream));
    ops->launches += sums ? 2 : 1;
    return EGERIA_OK;
}

// ---------------------------------------------------------------- AdamW
size_t egeria_adamw_workspace_bytes(int count, const egeria_adamw_tensor *tensors, uint32_t flags) {
    if (count < 1 || !tensors || (flags & ~EGERIA_ADAMW_8BIT)) return 0;
    AdamLayout L;
    return adam_layout(count, tensors, L) ? L.total : 0;
}

egeria_status egeria_adamw_create(egeria_adamw **out, int count, const egeria_adamw_tensor *tensors, const void *const *grads,
                                  int32_t *steps, void *workspace, size_t workspace_bytes, uint32_t flags) {
    if (!out) return EGERIA_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 1 || !tensors || !grads || !steps || !aligned(steps, 4) || (flags & ~EGERIA_ADAMW_8BIT)) return EGERIA_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i)
        if (!good_adam_tensor(tensors[i], flags) || (tensors[i].n > 0 && (!grads[i] || !aligned(grads[i], size_of(tensors[i].grad_type)))))
            return EGERIA_ERR_INVALID_ARG;
    AdamLayout L;
    if (!adam_layout(count, tensors, L)) return EGERIA_ERR_UNSUPPORTED_SHAPE;
    if (!workspace || !aligned(workspace, EGERIA_WORKSPACE_ALIGN) || workspace_bytes < L.total) return EGERIA_ERR_WORKSPACE;
    int sms = 0;
    egeria_status s = device_ready(&sms);
    if (s != EGERIA_OK) return s;
    egeria_adamw *h = nullptr;
    try {
        h = new egeria_adamw();
        h->ws = static_cast<uint8_t *>(workspace);
        h->L = L;
        h->count = count;
        const bool small = (flags & EGERIA_ADAMW_8BIT) != 0;
        std::vector<uint8_t> image(L.total, 0);
        AdamTensor *tab = reinterpret_cast<AdamTensor *>(image.data() + L.tensors);
        int2 *chunks = reinterpret_cast<int2 *>(image.data() + L.chunks);
        memcpy(image.data() + L.grads, grads, (size_t)count * sizeof(void *));
        int64_t n_tab = 0, n_chunks = 0;
        for (int k = 0; k < kAdamClasses; ++k) {
            const int64_t tab0 = n_tab, chunk0 = n_chunks;
            const egeria_adamw_tensor *any = nullptr;
            for (int i = 0; i < count; ++i) {
                const egeria_adamw_tensor &t = tensors[i];
                if (adam_class(t) != k) continue;
                any = &t;
                AdamTensor &a = tab[n_tab];
                a.p = t.param, a.master = t.master, a.m = t.m, a.v = t.v, a.m_scale = t.m_scale, a.v_scale = t.v_scale;
                a.n = t.n, a.wd = t.weight_decay, a.module = t.module, a.index = i;
                const size_t moment = small ? 8 : 32;
                a.vector = aligned(t.param, 8 * size_of(t.param_type)) && aligned(t.master, 32) && aligned(t.m, moment) && aligned(t.v, moment);
                for (int64_t c = 0; c * kAdamChunk < t.n; ++c) chunks[n_chunks++] = make_int2((int)(n_tab - tab0), (int)c);
                ++n_tab;
            }
            if (!any) continue;
            egeria_adamw::Class c{};
            c.kernel = small ? adam_kernel<true>(any->param_type, any->grad_type, any->master != nullptr)
                             : adam_kernel<false>(any->param_type, any->grad_type, any->master != nullptr);
            int per_sm = 0;
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, c.kernel, kAdamThreads, 0) != cudaSuccess || per_sm < 1) {
                (void)cudaGetLastError();
                delete h;
                return EGERIA_ERR_CUDA;
            }
            c.params.tensors = reinterpret_cast<const AdamTensor *>(h->ws + L.tensors) + tab0;
            c.params.chunks = reinterpret_cast<const int2 *>(h->ws + L.chunks) + chunk0;
            c.params.grads = reinterpret_cast<const void *const *>(h->ws + L.grads);
            c.params.steps = steps;
            c.params.status = reinterpret_cast<int32_t *>(h->ws);
            c.params.ticket = reinterpret_cast<int32_t *>(h->ws + 128 * (1 + k));
            c.params.n_chunks = (int32_t)(n_chunks - chunk0);
            c.params.n_tensors = (int32_t)(n_tab - tab0);
            c.params.n_grads = count;
            c.grid = (int)std::max<int64_t>(1, std::min<int64_t>(n_chunks - chunk0, (int64_t)per_sm * sms));
            h->classes.push_back(c);
        }
        for (int i = 0; i < count; ++i) h->grad_size.push_back(tensors[i].n ? size_of(tensors[i].grad_type) : 0);
        // (first what was enqueued before: it may still write to this memory, and the copy would not wait for it)
        if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(h->ws, image.data(), L.total, cudaMemcpyHostToDevice) != cudaSuccess ||
            cudaDeviceSynchronize() != cudaSuccess) {
            (void)cudaGetLastError();
            delete h;
            return EGERIA_ERR_CUDA;
        }
    } catch (...) {  // out of host memory
        delete h;
        return EGERIA_ERR_INVALID_ARG;
    }
    *out = h;
    return EGERIA_OK;
}
egeria_status egeria_adamw_destroy(egeria_adamw *adamw) {
    if (!adamw) return EGERIA_ERR_INVALID_ARG;
    delete adamw;
    return EGERIA_OK;
}

egeria_status egeria_adamw_set_grads(egeria_adamw *adamw, void *cuda_stream, const void *const *grads) {
    if (!adamw || !grads) return EGERIA_ERR_INVALID_ARG;
    for (int i = 0; i < adamw->count; ++i)
        if (adamw->grad_size[i] && (!grads[i] || !aligned(grads[i], adamw->grad_size[i]))) return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    EGO_CUDA(cudaStreamIsCapturing(stream, &capturing));
    if (capturing != cudaStreamCaptureStatusNone) return EGERIA_ERR_INVALID_ARG;
    // ordinary (pageable) memory: the runtime stages the copy before it returns
    EGO_CUDA(cudaMemcpyAsync(adamw->ws + adamw->L.grads, grads, (size_t)adamw->count * sizeof(void *), cudaMemcpyHostToDevice, stream));
    adamw->last_stream = stream;
    return EGERIA_OK;
}

egeria_status egeria_adamw_step(egeria_adamw *adamw, void *cuda_stream, double lr, double beta1, double beta2, double eps,
                                const float *grad_scale, const uint8_t *frozen) {
    if (!adamw || !(lr >= 0.0) || !std::isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) ||
        !std::isfinite(eps) || !aligned(grad_scale, 4))
        return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    adamw->last_stream = stream;
    for (const egeria_adamw::Class &c : adamw->classes) {
        AdamParams p = c.params;
        p.frozen = frozen;
        p.grad_scale = grad_scale;
        p.lr = (float)lr;
        p.beta1 = (float)beta1, p.beta2 = (float)beta2;
        p.rest1 = (float)(1.0 - beta1), p.rest2 = (float)(1.0 - beta2);
        p.eps = (float)eps;
        p.ln_beta1 = std::log(beta1), p.ln_beta2 = std::log(beta2);
        EGO_CUDA(launch(c.kernel, dim3(c.grid), kAdamThreads, 0, stream, 1, p));
        ++adamw->launches;
    }
    return EGERIA_OK;
}

egeria_status egeria_adamw_device_status(egeria_adamw *adamw) {
    if (!adamw) return EGERIA_ERR_INVALID_ARG;
    EGO_CUDA(cudaStreamSynchronize(adamw->last_stream));
    int32_t v = 0;
    EGO_CUDA(cudaMemcpy(&v, adamw->ws, sizeof(v), cudaMemcpyDeviceToHost));
    if (v == 0) return EGERIA_OK;
    EGO_CUDA(cudaMemsetAsync(adamw->ws, 0, 128, adamw->last_stream));
    EGO_CUDA(cudaStreamSynchronize(adamw->last_stream));
    return static_cast<egeria_status>(v);
}
int64_t egeria_adamw_launch_count(const egeria_adamw *adamw) { return adamw ? adamw->launches : 0; }

}  // extern "C"
