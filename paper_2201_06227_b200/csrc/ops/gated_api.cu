// Host side of the gated feed-forward blocks (include/egeria_ops.h): argument checks, plans, launches.
#include "ops_host.h"

namespace egeria {
namespace ops {

// ---------------------------------------------------------------- kernels
template <typename T, int MODE>
static cudaError_t allow_mode() {
    cudaError_t e = allow_smem<T, 64, 1, 1, MODE>();
    if (e == cudaSuccess) e = allow_smem<T, 128, 1, 1, MODE>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 2, 1, MODE>();
    return e;
}
template <typename T>
static cudaError_t allow_store() {
    cudaError_t e = allow_smem<T, 128, 1, 1, kModeStore>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 2, 1, kModeStore>();
    if (e == cudaSuccess) e = allow_smem<T, 256, 2, 2, kModeStore>();
    return e;
}
template <typename T, int ROWS>
static cudaError_t allow_few() {
    cudaError_t e = cudaFuncSetAttribute(gated_few_kernel<T, ROWS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gated_few_kernel<T, ROWS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    return e;
}
template <typename T>
static cudaError_t allow_type() {
    cudaError_t e = allow_mode<T, kModeGated>();
    if (e == cudaSuccess) e = allow_mode<T, kModeGatedBack>();
    if (e == cudaSuccess) e = allow_store<T>();
    if (e == cudaSuccess) e = allow_few<T, 1>();
    if (e == cudaSuccess) e = allow_few<T, 2>();
    if (e == cudaSuccess) e = allow_few<T, 4>();
    return e;
}
// At a handle's first gated call (a captured one too): a process that makes none does not load these kernels (creation of its first handle
// 49 instead of 53 ms, 2 MB less on the device).
static cudaError_t allow_gated(egeria_ops *o) {
    if (o->gated) return cudaSuccess;
    cudaError_t e = allow_type<bf16>();
    if (e == cudaSuccess) e = allow_type<f16>();
    o->gated = e == cudaSuccess;
    return e;
}

template <typename T, int MODE>
static cudaError_t launch_type(const GemmPlan &g, const GemmParams<MODE> &p, int ctas, cudaStream_t stream) {
    if constexpr (MODE == kModeStore) {
        if (g.mb == 2) return launch_gemm<T, 256, 2, 2, MODE>(p, ctas, stream);
    } else {
        if (g.bn == 64) return launch_gemm<T, 64, 1, 1, MODE>(p, ctas, stream);
    }
    return g.cg == 2 ? launch_gemm<T, 256, 2, 1, MODE>(p, ctas, stream) : launch_gemm<T, 128, 1, 1, MODE>(p, ctas, stream);
}
template <int MODE>
static egeria_status launch_mode(egeria_ops *o, cudaStream_t stream, int type, const GemmPlan &g, const GemmParams<MODE> &p, int ctas) {
    EGO_CUDA((type == EGERIA_BF16 ? launch_type<bf16, MODE>(g, p, ctas, stream) : launch_type<f16, MODE>(g, p, ctas, stream)));
    ++o->launches;
    return EGERIA_OK;
}

// ---------------------------------------------------------------- plans
// A kind of tile, and the time of a unit of so many k blocks in cycles: a stage of 64 k takes the MMAs' cycles or its bytes at 43 a
// cycle, whichever is longer (seen at 8192 x 4096 x 8192: 10.2 TB/s from L2 to the SMs, 43 bytes a cycle for each, whatever else
// is idle).  Two accumulators of two tiles hide the shorter of products and epilogue, two of one tile about half of the epilogue.
struct Kind {
    int bn, cg, mb;
};
static double unit_cycles(const Kind &c, int64_t kblocks, double epilogue) {
    const double bytes = 128.0 * (128 * c.mb + c.bn / c.cg), per_block = std::max(2.0 * c.bn * c.mb, bytes / 43.0);
    const double products = per_block * (double)kblocks;
    return c.mb == 1 ? std::max(products, epilogue * c.bn) : products + epilogue * c.bn * c.mb * 0.5;
}
static GemmPlan with_tiles(const Kind &c, int64_t m, int64_t n, int splits) {
    const int rows = 128 * c.cg * c.mb;
    return GemmPlan{c.bn, c.cg, c.mb, splits, (int)((m + rows - 1) / rows), (int)((n + c.bn - 1) / c.bn)};
}
// One product with an epilogue of so many cycles per column; n in columns of the accumulator.  1024 -> 2816 hidden values, forward:
// 128 rows 22.3, 22.9 and 25.7 us with the three kinds, 256 rows 28.6, 24.2 and 26.6, 512 rows 38.7, 33.2 and 32.0; 16384 rows 328
// and 248 with the latter two, 266 with tiles of 512 x 256, whose epilogue nothing hides.
static GemmPlan plan_single(int64_t m, int64_t n, int64_t k, int sms, double epilogue) {
    constexpr Kind kinds[3] = {{64, 1, 1}, {128, 1, 1}, {256, 2, 1}};
    GemmPlan best{};
    double best_t = 1e300;
    for (const Kind &c : kinds) {
        const GemmPlan g = with_tiles(c, m, n, 1);
        const int64_t units = (int64_t)g.tiles_m * g.tiles_n, workers = sms / c.cg;
        const double t = (double)((units + workers - 1) / workers) * unit_cycles(c, (k + kGemmK - 1) / kGemmK, epilogue) + epilogue * c.bn +
                         (c.cg == 2 ? 600.0 : 0.0);
        if (t < best_t) best_t = t, best = g;
    }
    return best;
}
// Up to four products that are only stored.  Of several, all but the last sum over equally many k and are split alike.  Where the
// tiles suffice for it, 512 x 256 of them take a quarter less from L2 than 256 x 256 (16384 rows, 1024 and 2816 wide: 324 us for
// the four of a backward pass, 1457 TFLOP/s, against 372).
static void plan_store(const Product *jobs, int count, int sms, GemmPlan *plan) {
    constexpr Kind kinds[3] = {{128, 1, 1}, {256, 2, 1}, {256, 2, 2}};
    constexpr double epilogue = 6.0;
    auto blocks = [](const Product &j) { return (j.k + kGemmK - 1) / kGemmK + (j.k2 + kGemmK - 1) / kGemmK; };
    auto split_cycles = [](const Kind &c, int splits) { return splits > 1 ? 2500.0 + 4.0 * c.bn + 4.0 * c.bn * splits : 0.0; };
    double best_t = 1e300;
    const int lead = count > 1 ? count - 1 : 1;
    for (const Kind &c : kinds) {
        const int64_t workers = sms / c.cg, most = c.mb > 1 ? 1 : std::min(sms, kMaxSplitCtas) / c.cg;  // units of a split product at most
        // the last product by itself first
        GemmPlan last{};
        double rest = 0.0, tail = 0.0;
        if (count > 1) {
            double last_t = 1e300;
            const int64_t kb = blocks(jobs[lead]);
            for (int splits = 1; splits <= 64 && splits <= kb; ++splits) {
                const GemmPlan g = with_tiles(c, jobs[lead].m, jobs[lead].n, splits);
                const int64_t units = (int64_t)g.tiles_m * g.tiles_n * splits;
                if (splits > 1 && units > most) break;
                const double one = unit_cycles(c, (kb + splits - 1) / splits, epilogue), add = split_cycles(c, splits);
                const double t = (double)((units + workers - 1) / workers) * one + add;
                if (t < last_t) last_t = t, last = g, tail = one + add, rest = (double)units * one / (double)workers;
            }
        }
        const int64_t kb = blocks(jobs[0]);
        for (int splits = 1; splits <= 64 && splits <= kb; ++splits) {
            GemmPlan g[kMaxProblems];
            int64_t units = 0;
            bool fits = true;
            for (int i = 0; i < lead; ++i) {
                g[i] = with_tiles(c, jobs[i].m, jobs[i].n, splits);
                const int64_t n = (int64_t)g[i].tiles_m * g[i].tiles_n * splits;
                fits = fits && (splits == 1 || n <= most);
                units += n;
            }
            if (!fits) break;
            const double one = unit_cycles(c, (kb + splits - 1) / splits, epilogue);
            double t = (double)((units + workers - 1) / workers) * one;
            if (count > 1) t = std::max(t, (double)units * one / (double)workers + rest + 0.5 * tail);
            t += split_cycles(c, splits);
            if (t < best_t) {
                best_t = t;
                std::copy(g, g + lead, plan);
                if (count > 1) plan[lead] = last;
            }
        }
    }
}

// ---------------------------------------------------------------- workspace
struct GatedLayout {
    size_t part[4], x, w_gate, w_up, w_down, dy, h, dg, du, sums, sums2, sums_down, total;
};
static int64_t pad16(int64_t v) { return (v + 15) / 16 * 16; }
static int64_t gated_sums(int64_t rows, int64_t hidden) { return (rows + 31) / 32 * hidden; }
static GatedLayout gated_layout(int64_t rows, int64_t inp, int64_t hidden, int64_t out) {
    GatedLayout L;
    size_t off = kHeadBytes;
    // (the largest sizes' products leave 64 bits: no workspace has 2^62 bytes)
    auto take = [&](int64_t a, int64_t b, int size) {
        const size_t at = off;
        const unsigned __int128 end = (unsigned __int128)off + (unsigned __int128)a * (unsigned __int128)b * (unsigned)size;
        off = end > ((unsigned __int128)1 << 62) ? (size_t)1 << 62 : up((size_t)end, 1024);
        return at;
    };
    L.part[0] = take(1, (int64_t)std::max(split_bytes(rows, out, hidden), split_bytes(out, hidden, rows)), 1);  // y, or dw_down
    L.part[1] = take(1, (int64_t)split_bytes(hidden, inp, rows), 1);
    L.part[2] = take(1, (int64_t)split_bytes(hidden, inp, rows), 1);
    L.part[3] = take(1, (int64_t)split_bytes(rows, inp, 2 * hidden), 1);
    L.x = take(rows, pad8(inp), 2);
    L.w_gate = take(hidden, pad8(inp), 2);
    L.w_up = take(hidden, pad8(inp), 2);
    L.w_down = take(out, pad8(hidden), 2);
    L.dy = take(rows, pad8(out), 2);
    L.h = take(rows, pad16(hidden), 2);
    L.dg = take(rows, pad16(hidden), 2);
    L.du = take(rows, pad16(hidden), 2);
    L.sums = take((rows + 31) / 32, hidden, 4);
    L.sums2 = take((rows + 31) / 32, hidden, 4);
    L.sums_down = take(1, slope_sums(rows, out), 4);
    L.total = off;
    return L;
}
static egeria_status good_gated_sizes(int64_t rows, int64_t inp, int64_t hidden, int64_t out) {
    const egeria_status s = good_sizes(rows, inp, hidden);
    return s != EGERIA_OK ? s : good_sizes(rows, hidden, out);
}

// ---------------------------------------------------------------- a few rows
template <typename T, int ROWS>
static cudaError_t launch_few(const GatedEpilogue &e, const egeria_gated_forward_args &a, bool wide, int sms, cudaStream_t stream) {
    const int smem = ROWS * (int)((a.inp + 255) / 256 * 256) * 2;
    const int grid = (int)std::min<int64_t>((a.hidden + 7) / 8, (int64_t)sms * 4);
    const T *x = static_cast<const T *>(a.x), *g = static_cast<const T *>(a.w_gate), *u = static_cast<const T *>(a.w_up);
    return launch(wide ? gated_few_kernel<T, ROWS, true> : gated_few_kernel<T, ROWS, false>, dim3(grid), 256, smem, stream, 1, e, (int32_t)a.rows,
                  (int32_t)a.hidden, x, a.ldx, g, a.ldw_gate, u, a.ldw_up, (int32_t)a.inp);
}
template <typename T>
static cudaError_t launch_few_any(const GatedEpilogue &e, const egeria_gated_forward_args &a, bool wide, int sms, cudaStream_t stream) {
    if (a.rows <= 1) return launch_few<T, 1>(e, a, wide, sms, stream);
    if (a.rows <= 2) return launch_few<T, 2>(e, a, wide, sms, stream);
    return launch_few<T, 4>(e, a, wide, sms, stream);
}

template <typename T, int ROWS>
static cudaError_t launch_down(const Epilogue &e, const egeria_gated_forward_args &a, const T *h, int64_t ldh, bool wide, cudaStream_t stream) {
    const unsigned grid = (unsigned)((a.out + 8 / kDownWarps - 1) / (8 / kDownWarps));
    return launch(wide ? gated_down_few_kernel<T, ROWS, true> : gated_down_few_kernel<T, ROWS, false>, dim3(grid), 256, 0, stream, 1, e, (int32_t)a.rows,
                  (int32_t)a.out, h, ldh, static_cast<const T *>(a.w_down), a.ldw_down, (int32_t)a.hidden);
}
template <typename T>
static cudaError_t launch_down_any(const Epilogue &e, const egeria_gated_forward_args &a, const void *h, int64_t ldh, bool wide, cudaStream_t stream) {
    if (a.rows <= 1) return launch_down<T, 1>(e, a, static_cast<const T *>(h), ldh, wide, stream);
    if (a.rows <= 2) return launch_down<T, 2>(e, a, static_cast<const T *>(h), ldh, wide, stream);
    return launch_down<T, 4>(e, a, static_cast<const T *>(h), ldh, wide, stream);
}

// Whether any of the written matrices shares a value with another or with one that is read.
template <int W, int R>
static bool any_overlap(const Extent (&written)[W], const Extent (&read)[R]) {
    for (int i = 0; i < W; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(written[i], written[j])) return true;
        for (const Extent &r : read)
            if (overlap(written[i], r)) return true;
    }
    return false;
}

}  // namespace ops
}  // namespace egeria

using namespace egeria;
using namespace egeria::ops;

extern "C" {

size_t egeria_gated_workspace_bytes(int64_t rows, int64_t inp, int64_t hidden, int64_t out) {
    if (good_gated_sizes(rows, inp, hidden, out) != EGERIA_OK) return 0;
    return gated_layout(rows, inp, hidden, out).total;
}

egeria_status egeria_gated_forward(egeria_ops *ops, void *cuda_stream, const egeria_gated_forward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_gated_forward_args &a = *args;
    if ((a.type != EGERIA_BF16 && a.type != EGERIA_F16) || !good_act(a.act)) return EGERIA_ERR_INVALID_ARG;
    egeria_status s = good_gated_sizes(a.rows, a.inp, a.hidden, a.out);
    if (s != EGERIA_OK) return s;
    if (a.rows == 0) return EGERIA_OK;
    if (!good_matrix(a.x, a.ldx, a.inp, 2) || !good_matrix(a.w_gate, a.ldw_gate, a.inp, 2) || !good_matrix(a.w_up, a.ldw_up, a.inp, 2) ||
        !good_matrix(a.w_down, a.ldw_down, a.hidden, 2) || !good_matrix(a.y, a.ldy, a.out, 2) || !good_optional(a.residual, a.ldr, a.out, 2) ||
        !good_optional(a.g, a.ldg, a.hidden, 2) || !good_optional(a.u, a.ldu, a.hidden, 2) || !a.g != !a.u || !aligned(a.b_gate, 2) ||
        !aligned(a.b_up, 2) || !aligned(a.b_down, 2))
        return EGERIA_ERR_INVALID_ARG;
    const bool onto = a.residual == a.y && (a.ldr == a.ldy || a.rows == 1);
    const Extent written[3] = {{a.y, a.ldy, a.rows, a.out}, {a.g, a.ldg, a.rows, a.hidden}, {a.u, a.ldu, a.rows, a.hidden}};
    const Extent read[8] = {{a.x, a.ldx, a.rows, a.inp},           {a.w_gate, a.ldw_gate, a.hidden, a.inp}, {a.w_up, a.ldw_up, a.hidden, a.inp},
                            {a.w_down, a.ldw_down, a.out, a.hidden}, {a.b_gate, a.hidden, 1, a.hidden},     {a.b_up, a.hidden, 1, a.hidden},
                            {a.b_down, a.out, 1, a.out},           {onto ? nullptr : a.residual, a.ldr, a.rows, a.out}};
    if (any_overlap(written, read)) return EGERIA_ERR_INVALID_ARG;
    const GatedLayout L = gated_layout(a.rows, a.inp, a.hidden, a.out);
    if (ops->ws_bytes < L.total) return EGERIA_ERR_WORKSPACE;
    EGO_CUDA(allow_gated(ops));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    ops->last_stream = stream;

    GatedEpilogue e{};
    e.bias = a.b_gate;
    e.bias2 = a.b_up;
    e.out = ops->ws + L.h;
    e.ldo = pad16(a.hidden);
    e.z = a.g, e.ldz = a.ldg;
    e.z2 = a.u, e.ldz2 = a.ldu;
    e.act = a.act;
    egeria_linear_forward_args down{};
    down.type = a.type;
    down.rows = a.rows, down.inp = a.hidden, down.out = a.out;
    down.x = e.out, down.ldx = e.ldo;
    down.w = a.w_down, down.ldw = a.ldw_down;
    down.bias = a.b_down;
    down.residual = a.residual, down.ldr = a.ldr;
    down.y = a.y, down.ldy = a.ldy;
    const int few_rows = a.rows <= 2 ? (int)a.rows : 4;
    if (a.rows <= kFewRows && (a.inp + 255) / 256 * 256 * 2 * few_rows <= kFewSmem) {
        const bool wide = a.inp % 8 == 0 && a.ldw_gate % 8 == 0 && a.ldw_up % 8 == 0 && aligned(a.w_gate, 16) && aligned(a.w_up, 16);
        EGO_CUDA(a.type == EGERIA_BF16 ? launch_few_any<bf16>(e, a, wide, ops->sms, stream) : launch_few_any<f16>(e, a, wide, ops->sms, stream));
        ++ops->launches;
        Epilogue d{};
        d.bias = a.b_down;
        d.extra = a.residual, d.ldx = a.ldr;
        d.out = a.y, d.ldo = a.ldy;
        const bool wide_down = a.hidden % 8 == 0 && a.ldw_down % 8 == 0 && aligned(a.w_down, 16);
        EGO_CUDA(a.type == EGERIA_BF16 ? launch_down_any<bf16>(d, a, e.out, e.ldo, wide_down, stream)
                                       : launch_down_any<f16>(d, a, e.out, e.ldo, wide_down, stream));
        ++ops->launches;
        return EGERIA_OK;
    } else {
        PrepareParams prep{};
        prep.status = reinterpret_cast<int32_t *>(ops->ws);
        Product job{a.rows, a.hidden, a.inp, {a.x, a.ldx, a.rows, a.inp, false}, {a.w_gate, a.ldw_gate, a.hidden, a.inp, false}, e, 0};
        job.b2 = {a.w_up, a.ldw_up, a.hidden, a.inp, false};
        make_loadable(ops, job.a, L.x, prep.pack[0]);
        make_loadable(ops, job.b, L.w_gate, prep.pack[1]);
        make_loadable(ops, job.b2, L.w_up, prep.pack[2]);
        Operand w_down{a.w_down, a.ldw_down, a.out, a.hidden, false};  // of the second product: in the same launch
        make_loadable(ops, w_down, L.w_down, prep.pack[3]);
        down.w = w_down.p, down.ldw = w_down.ld;
        if ((s = run_prepare(ops, stream, a.type, prep, false)) != EGERIA_OK) return s;
        const GemmPlan g = plan_single(a.rows, 2 * a.hidden, a.inp, ops->sms, a.g ? 20.0 : 12.0);
        GemmParams<kModeGated> p;
        int ctas = 0;
        if ((s = fill_products(ops, a.type, &job, &g, 1, p, ctas)) != EGERIA_OK) return s;
        if ((s = launch_mode(ops, stream, a.type, g, p, ctas)) != EGERIA_OK) return s;
    }
    return linear_forward_at(ops, stream, down, L.part[0], 0, L.w_down);
}

egeria_status egeria_gated_backward(egeria_ops *ops, void *cuda_stream, const egeria_gated_backward_args *args) {
    if (!ops || !args) return EGERIA_ERR_INVALID_ARG;
    const egeria_gated_backward_args &a = *args;
    if ((a.type != EGERIA_BF16 && a.type != EGERIA_F16) || !good_act(a.act)) return EGERIA_ERR_INVALID_ARG;
    egeria_status s = good_gated_sizes(a.rows, a.inp, a.hidden, a.out);
    if (s != EGERIA_OK) return s;
    if (!good_optional(a.dx, a.lddx, a.inp, 2) || !good_optional(a.dw_gate, a.lddw_gate, a.inp, 2) || !good_optional(a.dw_up, a.lddw_up, a.inp, 2) ||
        !good_optional(a.dw_down, a.lddw_down, a.hidden, 2) || !aligned(a.db_gate, 2) || !aligned(a.db_up, 2) || !aligned(a.db_down, 2))
        return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (a.rows == 0) {
        ops->last_stream = stream;
        auto clear = [&](void *p, int64_t ld, int64_t cols, int64_t rows) {
            return p ? cudaMemset2DAsync(p, (size_t)ld * 2, 0, (size_t)cols * 2, (size_t)rows, stream) : cudaSuccess;
        };
        EGO_CUDA(clear(a.dw_gate, a.lddw_gate, a.inp, a.hidden));
        EGO_CUDA(clear(a.dw_up, a.lddw_up, a.inp, a.hidden));
        EGO_CUDA(clear(a.dw_down, a.lddw_down, a.hidden, a.out));
        EGO_CUDA(clear(a.db_gate, a.hidden, a.hidden, 1));
        EGO_CUDA(clear(a.db_up, a.hidden, a.hidden, 1));
        EGO_CUDA(clear(a.db_down, a.out, a.out, 1));
        return EGERIA_OK;
    }
    const bool gates = a.dx || a.dw_gate || a.dw_up || a.db_gate || a.db_up;  // what needs dg and du
    if (!good_matrix(a.dy, a.lddy, a.out, 2)) return EGERIA_ERR_INVALID_ARG;
    if ((gates || a.dw_down) && (!good_matrix(a.w_down, a.ldw_down, a.hidden, 2) || !good_matrix(a.g, a.ldg, a.hidden, 2) || !good_matrix(a.u, a.ldu, a.hidden, 2)))
        return EGERIA_ERR_INVALID_ARG;
    if ((a.dw_gate || a.dw_up) && !good_matrix(a.x, a.ldx, a.inp, 2)) return EGERIA_ERR_INVALID_ARG;
    if (a.dx && (!good_matrix(a.w_gate, a.ldw_gate, a.inp, 2) || !good_matrix(a.w_up, a.ldw_up, a.inp, 2))) return EGERIA_ERR_INVALID_ARG;
    const Extent written[7] = {{a.dx, a.lddx, a.rows, a.inp},          {a.dw_gate, a.lddw_gate, a.hidden, a.inp}, {a.dw_up, a.lddw_up, a.hidden, a.inp},
                               {a.dw_down, a.lddw_down, a.out, a.hidden}, {a.db_gate, a.hidden, 1, a.hidden},      {a.db_up, a.hidden, 1, a.hidden},
                               {a.db_down, a.out, 1, a.out}};
    const Extent read[7] = {{a.dy, a.lddy, a.rows, a.out},           {a.dw_gate || a.dw_up ? a.x : nullptr, a.ldx, a.rows, a.inp},
                            {a.dx ? a.w_gate : nullptr, a.ldw_gate, a.hidden, a.inp}, {a.dx ? a.w_up : nullptr, a.ldw_up, a.hidden, a.inp},
                            {gates || a.dw_down ? a.w_down : nullptr, a.ldw_down, a.out, a.hidden},
                            {gates || a.dw_down ? a.g : nullptr, a.ldg, a.rows, a.hidden}, {gates || a.dw_down ? a.u : nullptr, a.ldu, a.rows, a.hidden}};
    if (any_overlap(written, read)) return EGERIA_ERR_INVALID_ARG;
    const GatedLayout L = gated_layout(a.rows, a.inp, a.hidden, a.out);
    if (ops->ws_bytes < L.total) return EGERIA_ERR_WORKSPACE;
    EGO_CUDA(allow_gated(ops));
    ops->last_stream = stream;

    // dy as a tile load takes it, and its column sums
    Operand dy{a.dy, a.lddy, a.rows, a.out, false};
    const bool own_dy = (gates || a.dw_down) && (!aligned(a.dy, 16) || a.lddy % 8 != 0);
    if (own_dy) {
        dy.p = ops->ws + L.dy;
        dy.ld = pad8(a.out);
    }
    PrepareParams prep{};
    prep.status = reinterpret_cast<int32_t *>(ops->ws);
    ColumnSums sums[kMaxSums] = {};
    int n_sums = 0;
    bool wide = false;
    if (own_dy || a.db_down) {
        SlopeJob &j = prep.slope;
        j.dz = own_dy ? ops->ws + L.dy : nullptr;
        j.lddz = dy.ld;
        j.dy = a.dy;
        j.lddy = a.lddy;
        j.rows = a.rows;
        j.cols = (int32_t)a.out;
        j.strips = (int32_t)((a.out + 255) / 256);
        j.runs = slope_runs(a.rows, a.out);
        j.db = a.db_down;
        if (a.db_down) {
            j.sums = reinterpret_cast<float *>(ops->ws + L.sums_down);
            j.sums_room = slope_sums(a.rows, a.out);
            if (j.runs > 1) sums[n_sums++] = ColumnSums{j.sums, a.db_down, j.runs, j.cols};
        }
        wide = a.out % 8 == 0 && aligned(a.dy, 16) && a.lddy % 8 == 0;
    }
    Product back{}, jobs[kMaxProblems];
    int count = 0;
    if (gates || a.dw_down) {
        GatedEpilogue e{};
        e.extra = a.g, e.ldx = a.ldg;
        e.extra2 = a.u, e.ldx2 = a.ldu;
        e.out = ops->ws + L.dg, e.z = ops->ws + L.du;
        if (a.dw_down) e.z2 = ops->ws + L.h;
        e.ldo = e.ldz = e.ldz2 = pad16(a.hidden);
        e.act = a.act;
        if (a.db_gate || a.db_up) {
            e.sums = reinterpret_cast<float *>(ops->ws + L.sums);
            e.sums2 = reinterpret_cast<float *>(ops->ws + L.sums2);
            e.sums_room = gated_sums(a.rows, a.hidden);
            const int32_t n = (int32_t)((a.rows + 31) / 32), cols = (int32_t)a.hidden;
            if (a.db_gate) sums[n_sums++] = ColumnSums{e.sums, a.db_gate, n, cols};
            if (a.db_up) sums[n_sums++] = ColumnSums{e.sums2, a.db_up, n, cols};
        }
        back = Product{a.rows, a.hidden, a.out, dy, {a.w_down, a.ldw_down, a.out, a.hidden, true}, e, 0};
        make_loadable(ops, back.b, L.w_down, prep.pack[0]);
    }
    const Operand dg{ops->ws + L.dg, pad16(a.hidden), a.rows, a.hidden, false}, du{ops->ws + L.du, pad16(a.hidden), a.rows, a.hidden, false};
    auto turned = [](Operand o) {
        o.mn = true;
        return o;
    };
    auto store = [&](void *to, int64_t ld, int64_t m, int64_t n, int64_t k, const Operand &p, const Operand &q, size_t part) -> Product & {
        Product &j = jobs[count++] = Product{m, n, k, p, q, {}, part};
        j.epi.out = to;
        j.epi.ldo = ld;
        return j;
    };
    Operand x{a.x, a.ldx, a.rows, a.inp, true};
    if (a.dw_gate || a.dw_up) make_loadable(ops, x, L.x, prep.pack[1]);
    if (a.dw_gate) store(a.dw_gate, a.lddw_gate, a.hidden, a.inp, a.rows, turned(dg), x, L.part[1]);
    if (a.dw_up) store(a.dw_up, a.lddw_up, a.hidden, a.inp, a.rows, turned(du), x, L.part[2]);
    if (a.dw_down) store(a.dw_down, a.lddw_down, a.out, a.hidden, a.rows, turned(dy), {ops->ws + L.h, pad16(a.hidden), a.rows, a.hidden, true}, L.part[0]);
    if (a.dx) {
        Product &j = store(a.dx, a.lddx, a.rows, a.inp, a.hidden, dg, {a.w_gate, a.ldw_gate, a.hidden, a.inp, true}, L.part[3]);
        j.k2 = a.hidden;
        j.a2 = du;
        j.b2 = {a.w_up, a.ldw_up, a.hidden, a.inp, true};
        make_loadable(ops, j.b, L.w_gate, prep.pack[2]);
        make_loadable(ops, j.b2, L.w_up, prep.pack[3]);
    }
    if ((s = run_prepare(ops, stream, a.type, prep, wide)) != EGERIA_OK) return s;
    int ctas = 0;
    if (gates || a.dw_down) {
        GemmParams<kModeGatedBack> p;
        const GemmPlan g = plan_single(a.rows, a.hidden, a.out, ops->sms, 30.0);
        if ((s = fill_products(ops, a.type, &back, &g, 1, p, ctas)) != EGERIA_OK) return s;
        if ((s = launch_mode(ops, stream, a.type, g, p, ctas)) != EGERIA_OK) return s;
    }
    if (count) {
        GemmPlan plan[kMaxProblems];
        plan_store(jobs, count, ops->sms, plan);
        GemmParams<kModeStore> p;
        if ((s = fill_products(ops, a.type, jobs, plan, count, p, ctas)) != EGERIA_OK) return s;
        std::copy(sums, sums + kMaxSums, p.sums);
        return launch_mode(ops, stream, a.type, plan[0], p, ctas);
    }
    for (int i = 0; i < n_sums; ++i) {
        const dim3 grid((unsigned)((sums[i].cols + 31) / 32));
        EGO_CUDA(a.type == EGERIA_BF16 ? launch(add_columns_kernel<bf16>, grid, 512, 0, stream, 1, sums[i])
                                       : launch(add_columns_kernel<f16>, grid, 512, 0, stream, 1, sums[i]));
        ++ops->launches;
    }
    return EGERIA_OK;
}

}  // extern "C"
