// Host side of the Muon step (include/egeria_ops.h): argument checks, the list of units, launches.
#include <algorithm>
#include <cmath>
#include <iterator>
#include <new>
#include <utility>
#include <vector>

#include "muon.cuh"
#include "ops_host.h"

namespace egeria {
namespace ops {

constexpr int64_t kMuonMaxSide = (int64_t)1 << 22;

static bool good_muon_tensor(const egeria_muon_tensor &t) {
    if (t.rows < 0 || t.cols < 0 || t.param_type < EGERIA_F32 || t.param_type > EGERIA_F16 || t.module < -1) return false;
    if (t.grad_type != EGERIA_F32 && t.grad_type != t.param_type) return false;
    if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay) || !std::isfinite(t.scale)) return false;
    if (t.rows == 0 || t.cols == 0) return true;
    return t.param && t.m && aligned(t.param, size_of(t.param_type)) && aligned(t.master, 4) && aligned(t.m, 4);
}

// The ranges of addresses that a step writes, in order; false if two of them share a byte: a matrix that stands in the list twice would be
// updated from two workers at a time.  (The sides are within kMuonMaxSide here.)
using MuonRanges = std::vector<std::pair<uintptr_t, uintptr_t>>;
static bool muon_written(int count, const egeria_muon_tensor *t, MuonRanges &written) {
    written.clear();
    auto add = [&](const void *p, int64_t bytes) {
        if (p && bytes > 0) written.emplace_back(reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes);
    };
    for (int i = 0; i < count; ++i) {
        const int64_t n = t[i].rows * t[i].cols;
        add(t[i].param, n * (int64_t)size_of(t[i].param_type));
        add(t[i].master, n * 4);
        add(t[i].m, n * 4);
    }
    std::sort(written.begin(), written.end());
    for (size_t i = 1; i < written.size(); ++i)
        if (written[i].first < written[i - 1].second) return false;
    return true;
}
// Whether any of these bytes is among them.  (A gradient is read twice, once the momenta are written, and others' weights may be by then.)
static bool muon_meets(const MuonRanges &written, const void *p, int64_t bytes) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p), end = from + (uintptr_t)bytes;
    const auto next = std::lower_bound(written.begin(), written.end(), std::make_pair(from, (uintptr_t)0));
    return (next != written.end() && next->first < end) || (next != written.begin() && std::prev(next)->second > from);
}
static bool muon_small(const egeria_muon_tensor &t) {
    return std::min(t.rows, t.cols) <= kSmallSide && std::max(t.rows, t.cols) <= kSmallPanels * 64;
}
// Where things lie in the workspace.  The matrices' own part goes by their sides alone.
struct MuonPlaces {
    size_t x[2], lo, gram, poly, sums;
};
struct MuonLayout {
    size_t matrices, maps, grads, pieces, units, done, total;
    int64_t n_matrices, n_pieces, n_units;
    std::vector<int> which;           // the matrices that are not empty, the small ones last
    std::vector<MuonPlaces> places;   // theirs
    int large;                        // how many are not small
};
static int64_t up32(int64_t v) { return (v + 31) / 32 * 32; }
// Products of a tile: which columns of tiles a row of them has to take.  Of a symmetric product only those that reach the diagonal.
template <typename F>
static void muon_tiles(int64_t m, int64_t n, bool symmetric, int tile_rows, int bn, F each) {
    for (int64_t tm = 0; tm * tile_rows < m; ++tm)
        for (int64_t tn = symmetric ? tm * tile_rows / bn : 0; tn * bn < n; ++tn) each((int32_t)tm, (int32_t)tn);
}
struct MuonKind {
    int bn, cg;
};
// 256 x 256 tiles of a pair of CTAs where they go round all of them a few times, else 128 x 128: 54 convolutions of 16 to 64 channels (108
// tiles of 256) 100 us with the small ones and 131 with the large, 12 matrices of 333 x 333 and 333 x 1332 203 and 263.
static MuonKind muon_kind(int count, const egeria_muon_tensor *t) {
    int64_t tiles = 0;
    for (int i = 0; i < count; ++i)
        if (!muon_small(t[i])) tiles += ((t[i].rows + 255) / 256) * ((t[i].cols + 255) / 256);
    return tiles >= 2 * kSms ? MuonKind{256, 2} : MuonKind{128, 1};
}
static bool muon_layout(int count, const egeria_muon_tensor *t, int steps, MuonLayout &L) {
    for (int i = 0; i < count; ++i)
        if (t[i].rows > kMuonMaxSide || t[i].cols > kMuonMaxSide) return false;
    const MuonKind kind = muon_kind(count, t);
    L.n_matrices = L.n_pieces = L.n_units = 0;
    L.total = 256;  // status words
    L.places.clear();
    auto take = [&](int64_t n) {
        const size_t at = L.total;
        L.total = up(L.total + (size_t)n, 1024);
        return at;
    };
    L.which.clear();
    for (const bool small : {false, true}) {
        for (int i = 0; i < count; ++i)
            if (t[i].rows > 0 && t[i].cols > 0 && muon_small(t[i]) == small) L.which.push_back(i);
        if (!small) L.large = (int)L.which.size();
    }
    for (const int i : L.which) {
        const int64_t rows = t[i].rows, cols = t[i].cols, d = std::min(rows, cols);
        ++L.n_matrices;
        if (muon_small(t[i])) {
            MuonPlaces q{};
            q.lo = take(kSmallSide * up(std::max(rows, cols), 64) * 2);
            L.places.push_back(q);
            continue;
        }
        const int64_t pieces = (rows * cols + kMuonPiece - 1) / kMuonPiece;
        L.n_pieces += pieces;
        const int64_t r = (d + 128 * kind.cg - 1) / (128 * kind.cg), c = (d + kind.bn - 1) / kind.bn;
        if (r * c > (1 << 24)) return false;
        int64_t units = 0;
        muon_tiles(d, d, true, 128 * kind.cg, kind.bn, [&](int32_t, int32_t) { ++units; });
        L.n_units += steps * (2 * units + ((rows + 128 * kind.cg - 1) / (128 * kind.cg)) * ((cols + kind.bn - 1) / kind.bn));
        if (L.n_units > (1 << 28) || L.n_pieces > 0x7fffffff || L.n_matrices >= 0x7fffff) return false;  // (what the units' entries hold)
        MuonPlaces q;
        q.x[0] = take(rows * up32(cols) * 2);
        q.x[1] = take(rows * up32(cols) * 2);
        q.lo = take(rows * up32(cols) * 2);
        q.gram = take(d * up32(d) * 2);
        q.poly = take(d * up32(d) * 2);
        q.sums = take(pieces * 8);
        L.places.push_back(q);
    }
    L.matrices = take(L.n_matrices * (int64_t)sizeof(MuonMatrix));
    L.maps = take(L.n_matrices * kMuonMaps * (int64_t)sizeof(CUtensorMap));
    L.grads = take((int64_t)count * (int64_t)sizeof(void *));
    L.pieces = take(L.n_pieces * (int64_t)sizeof(int2));
    L.units = take(L.n_units * (int64_t)sizeof(int4));
    L.done = take(L.n_matrices * 4 + 4);
    return true;
}

template <int BN, int CG, bool NARROW>
static cudaError_t muon_allow() {
    return cudaFuncSetAttribute(muon_products_kernel<BN, CG, NARROW>, cudaFuncAttributeMaxDynamicSharedMemorySize, MuonCfg<BN, CG>::kSmem);
}
static cudaError_t muon_allow_all() {
    cudaError_t e = muon_allow<256, 2, false>();
    if (e == cudaSuccess) e = muon_allow<256, 2, true>();
    if (e == cudaSuccess) e = muon_allow<128, 1, false>();
    if (e == cudaSuccess) e = muon_allow<128, 1, true>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(muon_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem);
    return e;
}
template <int BN, int CG>
static cudaError_t muon_launch(const MuonParams &p, int workers, bool narrow, cudaStream_t stream) {
    auto kernel = narrow ? muon_products_kernel<BN, CG, true> : muon_products_kernel<BN, CG, false>;
    return launch(kernel, dim3(workers * CG), MuonCfg<BN, CG>::kThreads, MuonCfg<BN, CG>::kSmem, stream, CG, p);
}

}  // namespace ops
}  // namespace egeria

using namespace egeria;
using namespace egeria::ops;

struct egeria_muon {
    uint8_t *ws = nullptr;
    size_t grads = 0, total = 0;
    MuonKind kind{};
    MuonParams params{};
    int workers = 0, count = 0;
    std::vector<size_t> grad_size;   // of a value, 0 for an empty matrix
    std::vector<int64_t> grad_bytes;
    MuonRanges written;
    int64_t launches = 0;
    cudaStream_t last_stream = nullptr;
    uint32_t stall_next = 0;
    bool narrow = false;             // some matrix takes no whole lines
};

extern "C" {

size_t egeria_muon_workspace_bytes(int count, const egeria_muon_tensor *tensors, int steps) {
    if (count < 1 || !tensors || steps < 1 || steps > EGERIA_MUON_MAX_STEPS) return 0;
    for (int i = 0; i < count; ++i)
        if (tensors[i].rows < 0 || tensors[i].cols < 0) return 0;
    try {
        MuonLayout L;
        return muon_layout(count, tensors, steps, L) ? L.total : 0;
    } catch (...) {
        return 0;
    }
}

egeria_status egeria_muon_create(egeria_muon **out, int count, const egeria_muon_tensor *tensors, const void *const *grads, int steps,
                                 void *workspace, size_t workspace_bytes) {
    if (!out) return EGERIA_ERR_INVALID_ARG;
    *out = nullptr;
    if (count < 1 || !tensors || !grads || steps < 1 || steps > EGERIA_MUON_MAX_STEPS) return EGERIA_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        const egeria_muon_tensor &t = tensors[i];
        if (!good_muon_tensor(t) || (t.rows > 0 && t.cols > 0 && (!grads[i] || !aligned(grads[i], size_of(t.grad_type))))) return EGERIA_ERR_INVALID_ARG;
    }
    egeria_muon *h = nullptr;
    try {
        MuonLayout L;
        if (!muon_layout(count, tensors, steps, L)) return EGERIA_ERR_UNSUPPORTED_SHAPE;
        if (!workspace || !aligned(workspace, EGERIA_WORKSPACE_ALIGN) || workspace_bytes < L.total) return EGERIA_ERR_WORKSPACE;
        MuonRanges written;
        if (!muon_written(count, tensors, written)) return EGERIA_ERR_INVALID_ARG;
        for (const int i : L.which)
            if (muon_meets(written, grads[i], tensors[i].rows * tensors[i].cols * (int64_t)size_of(tensors[i].grad_type))) return EGERIA_ERR_INVALID_ARG;
        int dev = 0, major = 0, sms = 0;
        EGO_CUDA(cudaGetDevice(&dev));
        EGO_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
        if (major != 10) return EGERIA_ERR_UNSUPPORTED_DEVICE;
        EGO_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess || !fn) {
            (void)cudaGetLastError();
            return EGERIA_ERR_CUDA;
        }
        const EncodeTiledFn encode = reinterpret_cast<EncodeTiledFn>(fn);
        const MuonKind kind = muon_kind(count, tensors);
        EGO_CUDA(muon_allow_all());
        const int workers = sms / kind.cg;

        h = new egeria_muon();
        uint8_t *ws = h->ws = static_cast<uint8_t *>(workspace);
        h->grads = L.grads;
        h->total = L.total;
        h->kind = kind;
        h->count = count;
        std::vector<MuonMatrix> matrices;
        std::vector<CUtensorMap> maps((size_t)L.n_matrices * kMuonMaps);
        std::vector<int2> pieces;
        h->written = std::move(written);
        for (int i = 0; i < count; ++i) {
            const int64_t n = tensors[i].rows * tensors[i].cols;
            h->grad_size.push_back(n > 0 ? size_of(tensors[i].grad_type) : 0);
            h->grad_bytes.push_back(n * (int64_t)size_of(tensors[i].grad_type));
        }
        for (const int i : L.which) {
            const egeria_muon_tensor &t = tensors[i];
            const int k = (int)matrices.size();
            const MuonPlaces &at = L.places[k];
            MuonMatrix q{};
            q.param = t.param, q.master = t.master, q.m = t.m;
            for (int s = 0; s < 2; ++s) q.x[s] = reinterpret_cast<uint16_t *>(ws + at.x[s]);
            q.lo = reinterpret_cast<uint16_t *>(ws + at.lo);
            q.gram = reinterpret_cast<uint16_t *>(ws + at.gram);
            q.poly = reinterpret_cast<uint16_t *>(ws + at.poly);
            q.sums = reinterpret_cast<double *>(ws + at.sums);
            q.rows = t.rows, q.cols = t.cols, q.ldx = up32(t.cols);
            q.d = (int32_t)std::min(t.rows, t.cols);
            q.ldd = (int32_t)up32(q.d);
            q.wd = t.weight_decay, q.scale = t.scale;
            // near the root of the longer side: rows of an orthogonal matrix then have values near 1, and none comes near 65504
            q.up = (float)(1 << std::min(14, (int)std::floor(0.5 * std::log2((double)std::max(t.rows, t.cols)))));
            q.down = 1.0f / q.up;
            q.module = t.module, q.index = i, q.param_type = t.param_type, q.grad_type = t.grad_type;
            q.tall = t.rows > t.cols;
            q.pieces = (int32_t)((t.rows * t.cols + kMuonPiece - 1) / kMuonPiece);
            // (the gradient may move: the kernels look at its alignment)
            q.vector = t.cols % 8 == 0 && aligned(t.param, 8 * size_of(t.param_type)) && aligned(t.master, 32) && aligned(t.m, 32);
            auto map = [&](int which, const uint16_t *p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
                cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
                cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
                return encode(&maps[(size_t)k * kMuonMaps + which], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<uint16_t *>(p), dims, strides, box, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
            };
            bool ok = true;
            for (int s = 0; s < 2 && !muon_small(t); ++s)
                ok = ok && map(kMapX0 + 2 * s, q.x[s], q.rows, q.cols, q.ldx, 128) && map(kMapX0N + 2 * s, q.x[s], q.rows, q.cols, q.ldx, 64);
            if (!muon_small(t)) ok = ok && map(kMapGram, q.gram, q.d, q.d, q.ldd, 128) && map(kMapPoly, q.poly, q.d, q.d, q.ldd, 128);
            if (!ok) {
                delete h;
                return EGERIA_ERR_CUDA;
            }
            h->narrow = h->narrow || (k < L.large && !q.vector);
            for (int s = 0; s < q.pieces && k < L.large; ++s) pieces.push_back(make_int2(k, s));
            matrices.push_back(q);
        }
        // The units, product by product over all matrices, large ones first, so that a unit's matrix has mostly finished the product
        // before.  (In groups whose products go round the workers two to eight times, which meet more of their values in L2, the
        // 24 blocks of width 1024 took 5.75 to 5.18 ms against 5.15: the waits at a group's ends cost more.)
        std::vector<int> order(L.large);
        for (size_t i = 0; i < order.size(); ++i) order[i] = (int)i;
        std::stable_sort(order.begin(), order.end(), [&](int a, int b) {
            const MuonMatrix &p = matrices[a], &q = matrices[b];
            return p.d != q.d ? p.d > q.d : p.rows * p.cols > q.rows * q.cols;
        });
        const int tile_rows = 128 * kind.cg;
        std::vector<int4> units;
        std::vector<int32_t> so_far(matrices.size(), 0);
        auto add = [&](int k, int product) {
            const MuonMatrix &q = matrices[k];
            const int part = product % 3;
            const int32_t need = so_far[k] * kind.cg;
            const int64_t m = part == 2 ? q.rows : q.d, n = part == 2 ? q.cols : q.d, sum = part == 0 ? std::max(q.rows, q.cols) : q.d;
            const int32_t kblocks = (int32_t)((sum + kGemmK - 1) / kGemmK);
            muon_tiles(m, n, part != 2, tile_rows, kind.bn, [&](int32_t tm, int32_t tn) {
                units.push_back(make_int4(q.tall ? k | INT32_MIN : k, tm | tn << 16, product | kblocks << 8, need));
                ++so_far[k];
            });
        };
        for (int product = 0; product < 3 * steps; ++product)
            for (const int k : order) add(k, product);
        MuonParams &p = h->params;
        p.matrices = reinterpret_cast<const MuonMatrix *>(ws + L.matrices);
        p.maps = reinterpret_cast<const CUtensorMap *>(ws + L.maps);
        p.units = reinterpret_cast<const int4 *>(ws + L.units);
        p.pieces = reinterpret_cast<const int2 *>(ws + L.pieces);
        p.grads = reinterpret_cast<const void *const *>(ws + L.grads);
        p.done = reinterpret_cast<int32_t *>(ws + L.done);
        p.ticket = p.done + L.n_matrices;
        p.status = reinterpret_cast<int32_t *>(ws);
        p.n_units = (int32_t)units.size();
        p.n_pieces = (int32_t)pieces.size();
        p.n_matrices = (int32_t)matrices.size();
        p.first_small = L.large;
        p.products = 3 * steps;
        p.early = p.n_units >= 3 * steps * 4 * workers;
        h->workers = (int)std::min<int64_t>(workers, std::max(p.n_units, 1));
        auto put = [&](size_t at, const void *from, size_t bytes) { return bytes ? cudaMemcpy(ws + at, from, bytes, cudaMemcpyHostToDevice) : cudaSuccess; };
        // (first what was enqueued before: it may still write to this memory, and the copies would not wait for it)
        if ((int64_t)units.size() != L.n_units || cudaDeviceSynchronize() != cudaSuccess || cudaMemset(ws, 0, 256) != cudaSuccess ||
            put(L.matrices, matrices.data(), matrices.size() * sizeof(MuonMatrix)) != cudaSuccess ||
            put(L.maps, maps.data(), maps.size() * sizeof(CUtensorMap)) != cudaSuccess || put(L.grads, grads, (size_t)count * sizeof(void *)) != cudaSuccess ||
            put(L.pieces, pieces.data(), pieces.size() * sizeof(int2)) != cudaSuccess || put(L.units, units.data(), units.size() * sizeof(int4)) != cudaSuccess ||
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
egeria_status egeria_muon_destroy(egeria_muon *muon) {
    if (!muon) return EGERIA_ERR_INVALID_ARG;
    delete muon;
    return EGERIA_OK;
}

egeria_status egeria_muon_set_grads(egeria_muon *muon, void *cuda_stream, const void *const *grads) {
    if (!muon || !grads) return EGERIA_ERR_INVALID_ARG;
    for (int i = 0; i < muon->count; ++i)
        if (muon->grad_size[i] && (!grads[i] || !aligned(grads[i], muon->grad_size[i]) || muon_meets(muon->written, grads[i], muon->grad_bytes[i])))
            return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    EGO_CUDA(cudaStreamIsCapturing(stream, &capturing));
    if (capturing != cudaStreamCaptureStatusNone) return EGERIA_ERR_INVALID_ARG;
    // ordinary (pageable) memory: the runtime stages the copy before it returns
    EGO_CUDA(cudaMemcpyAsync(muon->ws + muon->grads, grads, (size_t)muon->count * sizeof(void *), cudaMemcpyHostToDevice, stream));
    muon->last_stream = stream;
    return EGERIA_OK;
}

egeria_status egeria_muon_step(egeria_muon *muon, void *cuda_stream, double lr, double beta, int nesterov, double eps, const float *grad_scale,
                               const uint8_t *frozen) {
    if (!muon || !(lr >= 0.0) || !std::isfinite(lr) || !(beta >= 0.0 && beta < 1.0) || !(eps >= 1e-30) || !std::isfinite(eps) || !aligned(grad_scale, 4))
        return EGERIA_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    muon->last_stream = stream;
    MuonParams p = muon->params;
    p.grad_scale = grad_scale;
    p.frozen = frozen;
    p.lr = (float)lr;
    p.beta = (float)beta;
    p.rest = (float)(1.0 - beta);
    p.eps = (float)eps;
    p.nesterov = nesterov != 0;
    p.stall = muon->stall_next;
    p.wait_limit_ns = muon->stall_next ? kTestWaitLimitNs : kWaitLimitNs;
    muon->stall_next = 0;
    if (p.first_small > 0) {
        EGO_CUDA(launch(muon_momentum_kernel, dim3(p.n_pieces), kMuonThreads, 0, stream, 1, p));
        EGO_CUDA(launch(muon_normalize_kernel, dim3(p.n_pieces), kMuonThreads, 0, stream, 1, p));
        EGO_CUDA((muon->kind.cg == 2 ? muon_launch<256, 2>(p, muon->workers, muon->narrow, stream)
                                     : muon_launch<128, 1>(p, muon->workers, muon->narrow, stream)));
        muon->launches += 3;
    }
    if (p.n_matrices > p.first_small) {
        EGO_CUDA(launch(muon_small_kernel, dim3(p.n_matrices - p.first_small), kSmallThreads, kSmallSmem, stream, 1, p));
        ++muon->launches;
    }
    return EGERIA_OK;
}

egeria_status egeria_muon_device_status(egeria_muon *muon) {
    if (!muon) return EGERIA_ERR_INVALID_ARG;
    EGO_CUDA(cudaStreamSynchronize(muon->last_stream));
    int32_t v = 0;
    EGO_CUDA(cudaMemcpy(&v, muon->ws, sizeof(v), cudaMemcpyDeviceToHost));
    if (v == 0) return EGERIA_OK;
    EGO_CUDA(cudaMemsetAsync(muon->ws, 0, 256, muon->last_stream));
    EGO_CUDA(cudaStreamSynchronize(muon->last_stream));
    return static_cast<egeria_status>(v);
}
egeria_status egeria_muon_debug_stall_next(egeria_muon *muon, int kind) {
    if (!muon || kind < 0 || kind > 2) return EGERIA_ERR_INVALID_ARG;
    muon->stall_next = (uint32_t)kind;
    return EGERIA_OK;
}
int64_t egeria_muon_launch_count(const egeria_muon *muon) { return muon ? muon->launches : 0; }

}  // extern "C"
