// What the host sides of the training operators share: launches, plans of matrix products, handles, argument checks.
#pragma once
#include <algorithm>
#include <cstring>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../../include/egeria_ops.h"
#include "linear.cuh"

#define EGO_CUDA(x)                                   \
    do {                                              \
        if ((x) != cudaSuccess) {                     \
            (void)cudaGetLastError();                 \
            return EGERIA_ERR_CUDA;                   \
        }                                             \
    } while (0)

namespace egeria {
namespace ops {
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
}  // namespace ops
}  // namespace egeria

struct egeria_ops {
    uint8_t *ws = nullptr;
    size_t ws_bytes = 0;
    egeria::ops::EncodeTiledFn encode = nullptr;
    int sms = 0;
    int64_t launches = 0;
    cudaStream_t last_stream = nullptr;
    uint32_t stall_next = 0;  // test hook: give-up path of the next product
    bool gated = false;       // the gated blocks' kernels are ready
};

namespace egeria {
namespace ops {

constexpr size_t kAlign = 256;
constexpr size_t kHeadBytes = EGERIA_OPS_WORKSPACE_MIN;  // status word, then the tickets of split products
constexpr size_t kTicketOff = 256;
constexpr int kMaxTickets = (int)((kHeadBytes - kTicketOff) / 4);
constexpr int kMaxSplitCtas = 160;                       // CTAs' worth of partial tiles at most
constexpr uint64_t kWaitLimitNs = 2000000000ull;
constexpr uint64_t kTestWaitLimitNs = 1000000ull;        // of a launch under egeria_ops_debug_stall_next
constexpr int64_t kMaxSize = ((int64_t)1 << 31) - 1024;  // tile coordinates are 32-bit
constexpr int kSms = 148;                                // what workspaces are sized for

// Every kernel is launched as a programmatic dependent of the one before it in the stream: its blocks may take their
// places while that one's last blocks are running, and each waits for it (griddepcontrol.wait) before it touches memory.
template <typename... Params, typename... Args>
inline cudaError_t launch(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream, int cluster, const Args &...args) {
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    c.attrs = attr;
    c.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, args...);
}

inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int64_t pad8(int64_t v) { return (v + 7) / 8 * 8; }
inline bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t size_of(int type) { return type == EGERIA_F32 ? 4 : 2; }

// ---------------------------------------------------------------- which tile for which product
struct GemmPlan {
    int bn, cg, mb, splits, tiles_m, tiles_n;
};

// Time of a product of m x n x k in cycles, by a model whose terms are measured ones: a stage of 64 k takes the
// MMAs' 2 * BN cycles or its bytes at 64 per cycle, whichever is longer; the units go in waves; the epilogue of
// the last wave is not hidden; a split product pays for its partial sums' way through L2.
inline double gemm_cycles(const GemmPlan &g, int64_t kblocks, int sms) {
    const double stage_bytes = 128.0 * 128 + 128.0 * g.bn / g.cg;
    const double per_block = std::max(2.0 * g.bn, stage_bytes / 64.0);
    const int64_t units = (int64_t)g.tiles_m * g.tiles_n * g.splits, workers = sms / g.cg;
    const double waves = (double)((units + workers - 1) / workers);
    const double main_loop = (double)((kblocks + g.splits - 1) / g.splits) * per_block;
    const double epilogue = 6.0 * g.bn;
    double t = waves * std::max(main_loop, epilogue) + epilogue + (g.cg == 2 ? 600.0 : 0.0);
    if (g.splits > 1) t += 2500.0 + 4.0 * g.bn + 4.0 * g.bn * g.splits;
    return t;
}

// The best split of the sum for one kind of tile.
inline GemmPlan plan_tile(int64_t m, int64_t n, int64_t k, int sms, int bn, int cg) {
    const int64_t kblocks = (k + kGemmK - 1) / kGemmK;
    GemmPlan g{bn, cg, 1, 1, (int)((m + 128 * cg - 1) / (128 * cg)), (int)((n + bn - 1) / bn)}, best = g;
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n;
    double best_t = gemm_cycles(g, kblocks, sms);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(64, kblocks), std::min(sms, kMaxSplitCtas) / (tiles * cg));
    for (g.splits = 2; g.splits <= most; ++g.splits) {
        const double t = gemm_cycles(g, kblocks, sms);
        if (t < best_t) best_t = t, best = g;
    }
    return best;
}
inline GemmPlan plan_gemm(int64_t m, int64_t n, int64_t k, int sms) {
    GemmPlan best{};
    double best_t = 1e300;
    for (int cg = 1; cg <= 2; ++cg)
        for (int bn = cg == 2 ? 128 : 64; bn <= 256; bn *= 2) {
            const GemmPlan g = plan_tile(m, n, k, sms, bn, cg);
            const double t = gemm_cycles(g, (k + kGemmK - 1) / kGemmK, sms);
            if (t < best_t) best_t = t, best = g;
        }
    return best;
}
static_assert(kMaxProblems * kMaxSplitCtas * kEpiWarps <= kMaxTickets, "a ticket for every warp of every split tile of each product");

// Bytes of partial tiles that a product of these sizes, or of smaller ones, may need under any plan.  (A product of more
// tiles than CTAs is not split, but a smaller one in its place is: the bound must not fall as a size grows.)
inline size_t split_bytes(int64_t m, int64_t n, int64_t k) {
    const int64_t kblocks = std::min<int64_t>((k + kGemmK - 1) / kGemmK, 64);
    if (kblocks <= 1) return 0;
    const int64_t tiles = std::min<int64_t>(((m + 255) / 256) * 2 * ((n + 255) / 256), kMaxSplitCtas);  // of 128 x 256
    return (size_t)std::min<int64_t>(tiles * kblocks, kMaxSplitCtas) * 128 * 256 * 4;
}

// Runs of rows that dz and its column sums are cut into: four blocks per SM at most, 32 rows at least.
inline int slope_runs(int64_t rows, int64_t cols) {
    const int64_t strips = (cols + 255) / 256;
    return (int)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, 4 * kSms / strips));
}
// Values of their partial sums at most, for these sizes and all smaller ones (runs * cols <= 4 * kSms * 256 beyond one run).
inline int64_t slope_sums(int64_t rows, int64_t cols) { return std::max(cols, std::min<int64_t>((rows + 31) / 32 * cols, 4 * kSms * 256)); }

// ---------------------------------------------------------------- products of a launch
template <typename T, int BN, int CG, int MB, int MODE>
inline cudaError_t allow_smem() {
    return cudaFuncSetAttribute(gemm_kernel<T, BN, CG, MB, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmCfg<BN, CG, MB>::kSmem);
}
template <typename T, int BN, int CG, int MB, int MODE>
inline cudaError_t launch_gemm(const GemmParams<MODE> &p, int ctas, cudaStream_t stream) {
    return launch(gemm_kernel<T, BN, CG, MB, MODE>, dim3(ctas), GemmCfg<BN, CG, MB>::kThreads, GemmCfg<BN, CG, MB>::kSmem, stream, CG, p);
}

constexpr int kFewSmem = 96 * 1024;
constexpr int kFewRows = 4;   // rows that go without the tensor cores: at 1024 x 4096 3.7 us for one row, 6.5 for two, 9.0 for four, 10.0 on the tensor cores
struct Operand {
    const void *p;
    int64_t ld, rows, cols;
    bool mn;  // the product's m (n) axis is the consecutive one: cols = m (n), rows = k
};

inline egeria_status encode_operand(const egeria_ops *o, CUtensorMap *map, const Operand &a, int type, int box_rows) {
    cuuint64_t dims[2] = {(cuuint64_t)a.cols, (cuuint64_t)a.rows};
    cuuint64_t strides[1] = {(cuuint64_t)a.ld * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)(a.mn ? 64 : box_rows)};
    cuuint32_t one[2] = {1, 1};
    const CUresult r = o->encode(map, type == EGERIA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                                 const_cast<void *>(a.p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? EGERIA_OK : EGERIA_ERR_CUDA;
}

// Widest access that all of a product's epilogue matrices take: 2 = 32 bytes, 1 = 16 bytes, 0 = one value.
inline void set_widths(GatedEpilogue &e) {
    int w = 2;
    auto see = [&](const void *q, int64_t ld) {
        if (!q) return;
        if (!aligned(q, 32) || ld % 16) w = std::min(w, aligned(q, 16) && ld % 8 == 0 ? 1 : 0);
    };
    see(e.out, e.ldo);
    see(e.z, e.ldz);
    see(e.extra, e.ldx);
    see(e.z2, e.ldz2);
    see(e.extra2, e.ldx2);
    e.wide = w;
    e.wide_bias = aligned(e.bias, 16) && aligned(e.bias2, 16);
}

// One product D = A B^T of a launch; k = the length of the summed axis.
struct Product {
    int64_t m, n, k;
    Operand a, b;
    GatedEpilogue epi;
    size_t part;            // its partial tiles in the workspace
    int64_t k2 = 0;         // and a second product a2 b2^T of that length is added to it
    Operand a2{}, b2{};     // (kModeGated: b2 is the up projection's weight, k2 = 0)
};

// The parameters of a launch of these products under these plans, which share the kind of tile.  Of several, the last may have
// another length than the others.  sizes of partial tiles go by split_bytes.
template <int MODE>
inline egeria_status fill_products(egeria_ops *o, int type, const Product *jobs, const GemmPlan *plan, int count, GemmParams<MODE> &p, int &ctas) {
    const int bn = plan[0].bn, cg = plan[0].cg, mb = plan[0].mb, workers = o->sms / cg;
    memset(&p, 0, sizeof(p));
    int64_t units = 0, last = 0;
    for (int i = 0; i < count; ++i) {
        const Product &j = jobs[i];
        const GemmPlan &g = plan[i];
        GemmProblem &q = p.problem[i];
        if (g.splits > 1 && (mb > 1 || (size_t)g.tiles_m * g.tiles_n * g.splits * cg * 128 * bn * 4 > split_bytes(j.m, j.n, j.k + j.k2)))
            return EGERIA_ERR_WORKSPACE;
        const int b_rows = MODE == kModeGated ? bn / 2 : bn / cg;
        egeria_status s = encode_operand(o, &q.a, j.a, type, kGemmM);
        if (s == EGERIA_OK) s = encode_operand(o, &q.b, j.b, type, b_rows);
        if (s == EGERIA_OK && j.b2.p) s = encode_operand(o, &q.b2, j.b2, type, b_rows);
        if (s == EGERIA_OK && j.a2.p) s = encode_operand(o, &q.a2, j.a2, type, kGemmM);
        if (s != EGERIA_OK) return s;
        q.m = (int32_t)j.m;
        q.n = (int32_t)j.n;
        q.kb2 = (int32_t)((j.k + kGemmK - 1) / kGemmK);
        const int64_t kblocks = q.kb2 + (j.k2 + kGemmK - 1) / kGemmK;
        q.kblocks = (int32_t)kblocks;
        q.tiles_m = g.tiles_m;
        q.tiles_n = g.tiles_n;
        q.splits = g.splits;
        const int64_t n_units = (int64_t)g.tiles_m * g.tiles_n * g.splits;
        if (n_units > 0x3fffffff) return EGERIA_ERR_UNSUPPORTED_SHAPE;
        q.units = (int32_t)n_units;
        units += n_units;
        last = n_units;
        // a strip of B of at most 16 MB, so that it stays in L2 next to the rows of A that go by
        q.group_n = (int32_t)std::max<int64_t>(1, std::min<int64_t>(g.tiles_n, ((int64_t)16 << 20) / (2 * (j.k + j.k2) * bn)));
        q.a_mn = j.a.mn;
        q.b_mn = j.b.mn;
        q.epi = j.epi;
        set_widths(q.epi);
        q.partials = reinterpret_cast<float *>(o->ws + j.part);
        q.tickets = reinterpret_cast<int32_t *>(o->ws + kTicketOff) + i * (kMaxTickets / kMaxProblems);
        q.partial_floats = (int64_t)split_bytes(j.m, j.n, j.k + j.k2) / 4;
        q.ticket_room = kMaxTickets / kMaxProblems;
    }
    if (units > 0x7fffffff) return EGERIA_ERR_UNSUPPORTED_SHAPE;
    const int used = (int)std::min<int64_t>(units, workers);
    p.first = (int32_t)(count > 1 ? units - last : units);
    p.second = (int32_t)(units - p.first);
    if (count > 1) {
        // the workers without a last unit of the leading products have its time for units of the last
        const GemmProblem &a = p.problem[0], &b = p.problem[count - 1];
        if (p.first % used) p.fill = (a.kblocks / a.splits) / std::max(1, b.kblocks / b.splits);
        p.fill = std::min<int64_t>(p.fill, p.second / used + 1);
    }
    p.is_f16 = type == EGERIA_F16;
    p.status = reinterpret_cast<int32_t *>(o->ws);
    p.stall = o->stall_next;
    p.wait_limit_ns = o->stall_next ? kTestWaitLimitNs : kWaitLimitNs;
    o->stall_next = 0;
    ctas = used * cg;
    return EGERIA_OK;
}
// One or two products that the linear layers' kernels take, under the plan that suits both.
egeria_status run_products(egeria_ops *o, cudaStream_t stream, int type, Product *jobs, int count, const ColumnSums &sums);

// The operand as a tile load takes it: itself, or the copy that `job` makes of it at `spare` with a pitch of pad8(cols).
inline void make_loadable(egeria_ops *o, Operand &a, size_t spare, PackJob &job) {
    if (aligned(a.p, 16) && a.ld % 8 == 0) return;
    job.src = static_cast<const uint16_t *>(a.p);
    job.dst = reinterpret_cast<uint16_t *>(o->ws + spare);
    job.ld = a.ld;
    job.pitch = pad8(a.cols);
    job.rows = a.rows;
    job.cols = a.cols;
    job.strips = (int32_t)((a.cols + 255) / 256);
    job.blocks = job.strips * (int32_t)std::max<int64_t>(1, std::min<int64_t>((a.rows + 7) / 8, 8 * kSms / job.strips));
    a.p = job.dst;
    a.ld = job.pitch;
}

egeria_status run_prepare(egeria_ops *o, cudaStream_t stream, int type, const PrepareParams &p, bool wide);
// A linear layer's forward pass whose arguments have been checked; part, x, w: where its partial tiles and copies of its operands go.
egeria_status linear_forward_at(egeria_ops *o, cudaStream_t stream, const egeria_linear_forward_args &a, size_t part, size_t x, size_t w);

inline bool good_matrix(const void *p, int64_t ld, int64_t cols, size_t elem) { return p && aligned(p, elem) && ld >= cols; }
inline bool good_optional(const void *p, int64_t ld, int64_t cols, size_t elem) { return !p || good_matrix(p, ld, cols, elem); }

// Whether two matrices of 2-byte values share one.  Parts of one buffer may lie between each other's rows.
struct Extent {
    const void *p;
    int64_t ld, rows, cols;
};
inline bool overlap(const Extent &a, const Extent &b) {
    if (a.rows < b.rows) return overlap(b, a);
    if (!a.p || !b.p) return false;
    const int64_t at = (int64_t)(reinterpret_cast<uintptr_t>(b.p) / 2) - (int64_t)(reinterpret_cast<uintptr_t>(a.p) / 2);
    if (at >= (a.rows - 1) * a.ld + a.cols || -at >= (b.rows - 1) * b.ld + b.cols) return false;
    if (a.ld == b.ld && b.rows > 1) {
        // row r of b begins at column `col` of a's row `row` + r and may reach into the next one
        const int64_t col = (at % a.ld + a.ld) % a.ld, row = (at - col) / a.ld;
        auto meet = [&](int64_t first) { return first < a.rows && first + b.rows > 0; };
        return (col < a.cols && meet(row)) || (col + b.cols > a.ld && meet(row + 1));
    }
    for (int64_t r = 0; r < b.rows; ++r) {
        const int64_t from = at + r * b.ld, end = from + b.cols;  // rows of a that end behind `from` and begin before `end`
        const int64_t first = from < a.cols ? 0 : (from - a.cols) / a.ld + 1;
        if (end > 0 && first <= std::min(a.rows - 1, (end - 1) / a.ld)) return true;
    }
    return false;
}
inline bool good_act(int act) { return act >= EGERIA_ACT_NONE && act <= EGERIA_ACT_SILU; }
inline egeria_status good_sizes(int64_t rows, int64_t inp, int64_t out) {
    if (rows < 0 || inp < 1 || out < 1) return EGERIA_ERR_INVALID_ARG;
    return rows > kMaxSize || inp > kMaxSize || out > kMaxSize ? EGERIA_ERR_UNSUPPORTED_SHAPE : EGERIA_OK;
}


}  // namespace ops
}  // namespace egeria
