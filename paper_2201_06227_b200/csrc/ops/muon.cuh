// The Muon step of a model's matrices: momentum, orthogonalisation by Newton-Schulz products, update.
//
//   m = beta m + (1 - beta) g      t = beta m + (1 - beta) g (Nesterov) or m
//   X = t / max(|t|, eps)          `steps` times:  A = X X^T,  X = a X + (b A + c A^2) X
//   p = p (1 - lr wd) - lr scale X
//
// (a, b, c) = (3.4445, -4.7750, 2.0315) sends every singular value from (0, 1] to about 1 and none above 1.21.  A matrix that is
// taller than wide takes A = X^T X and X = a X + X (b A + c A^2), the same polynomial from its shorter side, without being
// transposed: the tensor cores take either axis of an operand as the consecutive one.
//
// Operands are f16, sums 32 bits.  All values are below 4 in size, where f16 has three bits more than bf16.  A and the
// polynomial P = a I + b A + c A^2 are rounded once each.  X is kept as two f16 values, the second what the first leaves (22 bits): the
// products take the first, and a times the second is added.  Without it X's rounding would lie across its null space too, which no
// product damps and every step multiplies by a: a 512 x 512 matrix of rank 32 is off by 1.5e-3 (2-norm of the difference
// over that of the result, from the formula in 64 bits), with X in one f16 value by 2.9e-2, in one bf16 value by 0.23; a matrix of
// independent normal values by 1.5e-3, 1.3e-3 and 1.1e-2.  X is held times a power of two, so that its values stay off f16's
// lower end.
//
// All products of all matrices are one launch: a list of units (a tile of one of the 3 `steps` products of one matrix), which the
// workers (CTAs, or pairs of them) take in turn from its head.  A unit waits until the units of its matrix's product before it are
// done, which a counter per matrix says; the list has several matrices' tiles of a product side by side, so that as a rule it is long
// done.  What a unit waits for stands before it in the list and has been taken by a block that runs, however many run at once.
// A and A^2 are symmetric: tiles below the diagonal are left out, and each block of 32 x 32 above it is stored twice.
#pragma once
#include "../../../include/egeria_ops.h"
#include "linear.cuh"

namespace egeria {
namespace ops {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr int kMuonPiece = 8192;     // values of a matrix that a block takes in the elementwise passes
constexpr int kMuonThreads = 256;
enum { kMapX0 = 0, kMapX0N, kMapX1, kMapX1N, kMapGram, kMapPoly, kMuonMaps };  // N: boxes of 64 x 64 for the other axis

struct MuonMatrix {
    void *param;
    float *master, *m;
    uint16_t *x[2], *lo, *gram, *poly;
    double *sums;                    // of t^2, one per piece
    int64_t rows, cols, ldx;
    int32_t d, ldd;                  // the shorter side, and the pitch of gram and poly
    float wd, scale, up, down;       // X is held times `up`; down = 1 / up
    int32_t module, index, param_type, grad_type;
    int32_t tall, pieces;
    int32_t vector;                  // all but the gradient takes eight values of a row at a time
};
struct MuonParams {
    const MuonMatrix *matrices;
    const CUtensorMap *maps;         // [matrix][kMuonMaps]
    const int4 *units;               // matrix | tall << 31, tm | tn << 16, product | k blocks << 8, what the matrix's counter has to reach
    const int2 *pieces;              // matrix, piece
    const void *const *grads;
    int32_t *done;                   // per matrix: tiles (of one CTA) that are stored; -1 for one that is left out
    int32_t *ticket;                 // units that have been taken
    int32_t *status;
    const float *grad_scale;
    const uint8_t *frozen;
    float lr, beta, rest, eps;
    int32_t nesterov, n_units, n_pieces, n_matrices, products;
    int32_t first_small;             // from here on matrices go through muon_small_kernel
    int32_t early;                   // units are taken while the one before is loaded
    uint32_t stall;
    uint64_t wait_limit_ns;
};

// ---------------------------------------------------------------- elementwise passes
__device__ __forceinline__ bool muon_skips(const MuonParams &p, const MuonMatrix &t) { return p.frozen && t.module >= 0 && p.frozen[t.module]; }
__device__ __forceinline__ bool muon_scale(const MuonParams &p, float &scale) {
    scale = p.grad_scale ? *p.grad_scale : 1.0f;
    return isfinite(scale);
}
// Whether the elementwise passes take eight values at a time.
__device__ __forceinline__ bool muon_vector(const MuonParams &p, const MuonMatrix &t) {
    const uintptr_t grad = reinterpret_cast<uintptr_t>(p.grads[t.index]);
    return t.vector && grad % (t.grad_type == EGERIA_F32 ? 32 : 16) == 0;
}
// Eight gradients (or moments) of a matrix: consecutive ones from value e on, or, where its rows are not whole eights or not aligned,
// kMuonThreads apart; those behind `end` count as 0.
template <bool VECTOR, int STRIDE = kMuonThreads, typename T>
__device__ __forceinline__ void muon_read(float (&v)[8], const T *p, int64_t e, int64_t end) {
    if (VECTOR) {
        Raw8<T> r;
        load8(r, p + e);
        unpack8(v, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e + i * STRIDE < end ? to_f32(p[e + i * STRIDE]) : 0.0f;
    }
}
template <bool VECTOR>
__device__ __forceinline__ void muon_grads(float (&g)[8], const void *grad, int type, int64_t e, int64_t end) {
    if (type == EGERIA_F32)
        muon_read<VECTOR>(g, static_cast<const float *>(grad), e, end);
    else if (type == EGERIA_BF16)
        muon_read<VECTOR>(g, static_cast<const bf16 *>(grad), e, end);
    else
        muon_read<VECTOR>(g, static_cast<const f16 *>(grad), e, end);
}
template <int THREADS = kMuonThreads>
__device__ __forceinline__ double block_sum(double v, double *part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += part[w];
    return v;
}

// The momentum, and the sum of t^2 of each piece (in 64 bits: neither tiny nor huge gradients leave the range).
template <bool VECTOR>
__device__ __forceinline__ double muon_momentum_piece(const MuonParams &p, const MuonMatrix &t, int64_t e0, float scale) {
    const int64_t n = t.rows * t.cols, end = min(n, e0 + kMuonPiece);
    const void *grad = p.grads[t.index];
    double sum = 0.0;
    for (int64_t e = e0 + threadIdx.x * (VECTOR ? 8 : 1); e < end; e += kMuonThreads * 8) {
        float g[8], m[8];
        muon_grads<VECTOR>(g, grad, t.grad_type, e, end);
        muon_read<VECTOR>(m, t.m, e, end);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] *= scale;
            m[i] = fmaf(p.beta, m[i], p.rest * g[i]);
            const float v = p.nesterov ? fmaf(p.beta, m[i], p.rest * g[i]) : m[i];
            sum = fma((double)v, (double)v, sum);
        }
        if (VECTOR) {
            store8(t.m + e, m);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (e + i * kMuonThreads < end) t.m[e + i * kMuonThreads] = m[i];
        }
    }
    return sum;
}
__global__ void __launch_bounds__(kMuonThreads) muon_momentum_kernel(const MuonParams p) {
    __shared__ double part[kMuonThreads / 32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.ticket = 0;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < p.n_matrices; i += kMuonThreads) p.done[i] = muon_skips(p, p.matrices[i]) ? -1 : 0;
    float scale;
    if (!muon_scale(p, scale)) return;
    const int2 piece = p.pieces[blockIdx.x];
    if (!eg_check(piece.x >= 0 && piece.x < p.n_matrices, p.status, kCheckMuonPiece, blockIdx.x)) return;
    const MuonMatrix &t = p.matrices[piece.x];
    if (muon_skips(p, t)) return;
    const int64_t e0 = (int64_t)piece.y * kMuonPiece;
    const double sum = muon_vector(p, t) ? muon_momentum_piece<true>(p, t, e0, scale) : muon_momentum_piece<false>(p, t, e0, scale);
    const double all = block_sum(sum, part);
    if (threadIdx.x == 0) t.sums[piece.y] = all;
}

// X = t / max(|t|, eps), as two f16 values.
__device__ __forceinline__ void muon_split(float v, f16 &hi, f16 &lo) {
    hi = from_f32<f16>(v);
    lo = from_f32<f16>(v - to_f32(hi));
}
template <bool VECTOR>
__device__ __forceinline__ void muon_normalize_piece(const MuonParams &p, const MuonMatrix &t, int64_t e0, float scale, float inv) {
    const int64_t n = t.rows * t.cols, end = min(n, e0 + kMuonPiece);
    const void *grad = p.grads[t.index];
    const int64_t r0 = e0 / t.cols;
    const uint32_t c0 = (uint32_t)(e0 - r0 * t.cols), cols = (uint32_t)t.cols;
    for (int64_t e = e0 + threadIdx.x * (VECTOR ? 8 : 1); e < end; e += kMuonThreads * 8) {
        float g[8], v[8];
        muon_read<VECTOR>(v, t.m, e, end);
        if (p.nesterov) {
            muon_grads<VECTOR>(g, grad, t.grad_type, e, end);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(p.beta, v[i], p.rest * (g[i] * scale));
        }
        const uint32_t at = c0 + (uint32_t)(e - e0);
        if (VECTOR) {  // whole eights of a row
            const uint32_t row = at / cols, col = at - row * cols;
            uint16_t *x = t.x[0] + (r0 + row) * t.ldx + col, *lo = t.lo + (r0 + row) * t.ldx + col;
            uint32_t h[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f16 h0, l0, h1, l1;
                muon_split(v[2 * i] * inv, h0, l0);
                muon_split(v[2 * i + 1] * inv, h1, l1);
                h[i] = (uint32_t)__half_as_ushort(h0) | (uint32_t)__half_as_ushort(h1) << 16;
                l[i] = (uint32_t)__half_as_ushort(l0) | (uint32_t)__half_as_ushort(l1) << 16;
            }
            *reinterpret_cast<uint4 *>(x) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4 *>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (e + i * kMuonThreads >= end) break;
                const uint32_t to = at + i * kMuonThreads, row = to / cols, col = to - row * cols;
                f16 h, l;
                muon_split(v[i] * inv, h, l);
                t.x[0][(r0 + row) * t.ldx + col] = __half_as_ushort(h);
                t.lo[(r0 + row) * t.ldx + col] = __half_as_ushort(l);
            }
        }
    }
}
__global__ void __launch_bounds__(kMuonThreads) muon_normalize_kernel(const MuonParams p) {
    __shared__ double part[kMuonThreads / 32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float scale;
    if (!muon_scale(p, scale)) return;
    const int2 piece = p.pieces[blockIdx.x];
    if (!eg_check(piece.x >= 0 && piece.x < p.n_matrices, p.status, kCheckMuonPiece, blockIdx.x)) return;
    const MuonMatrix &t = p.matrices[piece.x];
    if (muon_skips(p, t)) return;
    double sum = 0.0;
    for (int i = threadIdx.x; i < t.pieces; i += kMuonThreads) sum += t.sums[i];
    sum = block_sum(sum, part);
    const double norm = fmax(sqrt(sum), (double)p.eps);  // (a NaN among the gradients gives eps here, and is still in t)
    const float inv = (float)((double)t.up / norm);
    const int64_t e0 = (int64_t)piece.y * kMuonPiece;
    if (muon_vector(p, t))
        muon_normalize_piece<true>(p, t, e0, scale, inv);
    else
        muon_normalize_piece<false>(p, t, e0, scale, inv);
}

// ---------------------------------------------------------------- products
// A 32 x 32 piece of the matrices in the workspace, whose rows are padded to whole pieces.  They are written and read by
// different SMs within one launch.
__device__ __forceinline__ void muon_fetch(uint32_t (&r)[16], const uint16_t *base, int64_t ld, const Tile &t) {
    if (t.lane < t.rows && t.cols > 0) {
        const uint16_t *p = base + (t.row0 + t.lane) * ld + t.col0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ld.relaxed.gpu.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r[8 * i]), "=r"(r[8 * i + 1]), "=r"(r[8 * i + 2]), "=r"(r[8 * i + 3]), "=r"(r[8 * i + 4]), "=r"(r[8 * i + 5]),
                           "=r"(r[8 * i + 6]), "=r"(r[8 * i + 7])
                         : "l"(p + 16 * i)
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = 0u;
    }
}
// Rows of a warp's 32 x 32 piece (this lane's row, as 16 pairs) into its shared memory, from which they are stored by whole lines: a row
// takes COLS / 8 sixteens of bytes, which change places with the row so that neither side meets a bank twice.
template <int COLS>
__device__ __forceinline__ uint32_t stage_place(uint32_t row, uint32_t sixteen) {
    return COLS == 64 ? row * 128 + ((sixteen ^ (row & 7)) << 4) : row * 64 + ((sixteen ^ (row >> 1 & 3)) << 4);
}
template <int COLS>
__device__ __forceinline__ void stage_rows(uint32_t at, uint32_t first, const uint32_t (&r)[16], int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + stage_place<COLS>(lane, first + i)), "r"(r[4 * i]), "r"(r[4 * i + 1]),
                     "r"(r[4 * i + 2]), "r"(r[4 * i + 3])
                     : "memory");
}
// The mirror image of a piece: this lane's row becomes column `lane`.
__device__ __forceinline__ void stage_mirror(uint32_t at, const uint32_t (&r)[16], int lane) {
#pragma unroll
    for (int c = 0; c < 32; ++c) {
        const uint16_t v = (uint16_t)(c & 1 ? r[c >> 1] >> 16 : r[c >> 1] & 0xffffu);
        asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + stage_place<32>(c, lane >> 3) + (lane & 7) * 2), "h"(v) : "memory");
    }
}
// 32 staged rows of COLS values to a matrix in the workspace, at its first of `rows` rows and `cols` columns that are left (rows are padded to
// whole pieces there).
template <int COLS>
__device__ __forceinline__ void store_staged(uint32_t at, uint16_t *to, int64_t ld, int rows, int cols, int lane) {
    constexpr int kLanes = COLS / 8, kRows = 32 / kLanes;  // lanes of a row, rows at a time
    const int sixteen = lane % kLanes, row0 = lane / kLanes;
    if (sixteen * 8 >= cols) return;
    uint4 v[32 / kRows];
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                     : "r"(at + stage_place<COLS>(row0 + i * kRows, sixteen))
                     : "memory");
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i)
        if (row0 + i * kRows < rows) *reinterpret_cast<uint4 *>(to + (row0 + i * kRows) * ld + sixteen * 8) = v[i];
}

// p = p keep - step X of a piece.  Four values of a row per lane, eight lanes a row: what X's 32 rows in lanes become through the
// warp's shared memory.
template <typename T>
__device__ __forceinline__ void muon_weights(uint32_t (&r)[2][16], const MuonMatrix &q, const Tile &t) {
    const int64_t at = (t.row0 + (t.lane >> 3)) * q.cols + t.col0 + (t.lane & 7) * 4;
    if ((t.lane & 7) * 4 >= t.cols) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if ((t.lane >> 3) + 4 * i >= t.rows) break;
        if (q.master || sizeof(T) == 4) {
            const float *p = (q.master ? q.master : static_cast<const float *>(q.param)) + at + 4 * i * q.cols;
            const uint4 w = *reinterpret_cast<const uint4 *>(p);
            uint32_t *to = &r[i >> 2][(i & 3) * 4];
            to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const T *>(q.param) + at + 4 * i * q.cols);
            r[i >> 2][(i & 3) * 4] = w.x, r[i >> 2][(i & 3) * 4 + 1] = w.y;
        }
    }
}
template <typename T>
struct Four;
template <>
struct Four<float> {
    static __device__ __forceinline__ void read(float (&v)[4], uint32_t a, uint32_t b) {}
    static __device__ __forceinline__ void write(void *p, const float (&v)[4]) { *static_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <typename T>
struct Four {
    static __device__ __forceinline__ void read(float (&v)[4], uint32_t a, uint32_t b) {
        const float2 x = unpack2<T>(a), y = unpack2<T>(b);
        v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
    }
    static __device__ __forceinline__ void write(void *p, const float (&v)[4]) {
        *static_cast<uint2 *>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    }
};
constexpr int kUpdatePitch = 36;  // floats
template <typename T>
__device__ __forceinline__ void muon_update_wide(const MuonMatrix &q, const uint32_t (&r)[2][16], const float *stage, float keep, float step, const Tile &t) {
    if ((t.lane & 7) * 4 >= t.cols) return;
    const int64_t at = (t.row0 + (t.lane >> 3)) * q.cols + t.col0 + (t.lane & 7) * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = (t.lane >> 3) + 4 * i;
        if (row >= t.rows) break;
        const float4 x = *reinterpret_cast<const float4 *>(stage + row * kUpdatePitch + (t.lane & 7) * 4);
        float v[4];
        if (q.master || sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(r[i >> 2][(i & 3) * 4 + k]);
        } else {
            Four<T>::read(v, r[i >> 2][(i & 3) * 4], r[i >> 2][(i & 3) * 4 + 1]);
        }
        v[0] = fmaf(v[0], keep, -step * x.x), v[1] = fmaf(v[1], keep, -step * x.y);
        v[2] = fmaf(v[2], keep, -step * x.z), v[3] = fmaf(v[3], keep, -step * x.w);
        const int64_t to = at + 4 * i * q.cols;
        Four<T>::write(static_cast<T *>(q.param) + to, v);
        if (q.master) Four<float>::write(q.master + to, v);
    }
}
// The same value by value, where rows are not whole eights or not aligned: lane = column, eight rows on their way at a time.
template <typename T>
__device__ __forceinline__ void muon_update_narrow(T *param, float *master, int64_t cols, const float *stage, float keep, float step, int rows) {
#pragma unroll 1
    for (int row = 0; row < rows; row += 8) {
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (row + i < rows) w[i] = master ? master[(row + i) * cols] : to_f32(param[(row + i) * cols]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (row + i >= rows) break;
            const float v = fmaf(w[i], keep, -step * stage[(row + i) * kUpdatePitch]);
            param[(row + i) * cols] = from_f32<T>(v);
            if (master) master[(row + i) * cols] = v;
        }
    }
}
template <typename F>
__device__ __forceinline__ void with_type(int type, F go) {
    if (type == EGERIA_F32)
        go(float());
    else if (type == EGERIA_BF16)
        go(bf16());
    else
        go(f16());
}

__device__ __forceinline__ int32_t load_acquire(const int32_t *p) {
    int32_t v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Until the matrix's counter has come that far, but not for ever: 1; 0 if it gave up, -1 if the matrix is left out.
__device__ __forceinline__ int muon_wait(const int32_t *done, int32_t need, volatile int *abort_flag, uint64_t limit_ns) {
    const int32_t v = load_acquire(done);
    if (v < 0) return -1;
    if (v >= need) return 1;
    const uint64_t t0 = ptx::globaltimer_ns();
    while (load_acquire(done) < need) {
        if (*abort_flag) return 0;
        if (ptx::globaltimer_ns() - t0 > limit_ns) {
            *abort_flag = 1;
            return 0;
        }
    }
    return 1;
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// As the linear layers' kernel, with a stage less, 8 KB of shared memory for each of the epilogue's warps, a warp that says
// when a tile is stored, and one that takes the units.
template <int BN, int CG>
struct MuonCfg : GemmCfg<BN, CG, 1> {
    using Base = GemmCfg<BN, CG, 1>;
    static constexpr int kStages = 5;
    static constexpr int kWarpStaging = 8192;
    static constexpr int kThreads = Base::kThreads + 64;
    static constexpr int kSmem = 1024 + kStages * Base::kStageBytes + kEpiWarps * kWarpStaging + 512;
    static_assert(kSmem <= 227 * 1024 && Base::kStageBytes % 1024 == 0, "shared memory of a CTA, tiles on their boundary");
};

struct MuonUnit {
    int32_t matrix, tm, tn, product, kind, kblocks, need;
    bool tall;
    bool same;  // a tile on the diagonal of a symmetric product: its operands are the same rows
};
__device__ __forceinline__ MuonUnit muon_unit(const int4 &q) {
    MuonUnit g;
    g.matrix = q.x & 0x7fffffff;
    g.tall = q.x < 0;
    g.tm = q.y & 0xffff, g.tn = q.y >> 16 & 0xffff;
    g.product = q.z & 0xff, g.kblocks = (int32_t)((uint32_t)q.z >> 8);
    g.kind = g.product % 3;
    g.need = q.w;
    g.same = g.kind != 2 && g.tm == g.tn;
    return g;
}
// The units that a worker has taken and found ready, for its roles in both CTAs of a pair: the last kUnitRing of them.  One thread
// takes them, at most one beyond those whose loads have been asked for.  No role falls further behind: the stages hold the loads of
// five units at most, a unit's products need the accumulator of the unit two before it drained, and the epilogue does not begin a
// unit before the warp that makes tiles known has taken the one kUnitLag before it, which has then seen the one before that stored.
constexpr int kUnitRing = 16, kUnitLag = 3;
constexpr int kNoMoreUnits = 0x7fffffff;
// An entry goes as two words of 56 bits, each with the low 8 bits of its number plus one, by which a reader knows it.
template <int CG>
__device__ __forceinline__ void unit_publish(uint32_t ring, uint32_t other, const int4 &q, int32_t n) {
    const uint64_t tag = (uint64_t)(n + 1 & 0xff) << 56;
    const uint64_t a = tag | (uint64_t)(q.x < 0) << 55 | (uint64_t)((uint32_t)q.x & 0x7fffff) << 32 | (uint32_t)q.y;
    const uint64_t b = tag | (uint64_t)((uint32_t)q.z & 0x1ffffff) << 31 | (uint32_t)(q.w & 0x7fffffff);
    asm volatile("fence.acq_rel.cluster;" ::: "memory");  // what the unit waited for comes before its entry
#pragma unroll
    for (int r = 0; r < CG; ++r) {
        const uint32_t to = (r ? other : ring) + (uint32_t)(n % kUnitRing) * 16;
        asm volatile("st.relaxed.cluster.shared::cluster.b64 [%0], %1;" ::"r"(to), "l"(a) : "memory");
        asm volatile("st.relaxed.cluster.shared::cluster.b64 [%0], %1;" ::"r"(to + 8), "l"(b) : "memory");
    }
}
// A number of units that one thread of this CTA raises and another waits for.
__device__ __forceinline__ void units_raise(uint32_t at, int32_t n) { asm volatile("st.release.cta.shared::cta.s32 [%0], %1;" ::"r"(at), "r"(n) : "memory"); }
__device__ __forceinline__ bool units_wait(uint32_t at, int32_t n, volatile int *abort_flag, uint64_t limit_ns) {
    auto there = [&] {
        int32_t r;
        asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
        return r >= n;
    };
    if (there()) return true;
    const uint64_t t0 = ptx::globaltimer_ns();
    while (!there()) {
        if (*abort_flag) return false;
        if (ptx::globaltimer_ns() - t0 > limit_ns) {
            *abort_flag = 1;
            return false;
        }
    }
    return true;
}
// Unit n of the worker, once it is there; false at the end and where the wait runs out.  What the unit waited for has then been
// stored for this thread too.
__device__ __forceinline__ bool unit_next(MuonUnit &g, uint32_t ring, int32_t n, volatile int *abort_flag, uint64_t limit_ns) {
    const uint32_t at = ring + (uint32_t)(n % kUnitRing) * 16;
    const uint32_t tag = n + 1 & 0xff;
    uint64_t a, b;
    auto there = [&] {
        asm volatile("ld.acquire.cluster.shared::cta.b64 %0, [%1];" : "=l"(a) : "r"(at) : "memory");
        asm volatile("ld.acquire.cluster.shared::cta.b64 %0, [%1];" : "=l"(b) : "r"(at + 8) : "memory");
        return (uint32_t)(a >> 56) == tag && (uint32_t)(b >> 56) == tag;
    };
    bool ok = there();
    for (int i = 0; !ok && i < 64; ++i) ok = there();
    if (!ok) {
        const uint64_t t0 = ptx::globaltimer_ns();
        while (!there()) {
            if (*abort_flag) return false;
            if (ptx::globaltimer_ns() - t0 > limit_ns) {
                *abort_flag = 1;
                return false;
            }
        }
    }
    const uint32_t matrix = (uint32_t)(a >> 32) & 0x7fffff;
    if (matrix == 0x7fffff) return false;
    g = muon_unit(make_int4((int)(matrix | (a >> 55 & 1 ? 0x80000000u : 0u)), (int)(uint32_t)a, (int)(uint32_t)(b >> 31 & 0x1ffffff),
                            (int)(uint32_t)(b & 0x7fffffff)));
    return true;
}

// NARROW: some matrix's rows are not whole eights or not aligned (without that code the other matrices' takes fewer registers: 24 blocks of
// width 1024 5.00 instead of 5.17 ms).
template <int BN, int CG, bool NARROW>
__global__ void __launch_bounds__(MuonCfg<BN, CG>::kThreads, 1) muon_products_kernel(const __grid_constant__ MuonParams p) {
    using Cfg = MuonCfg<BN, CG>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    uint8_t *staging = smem + Cfg::kStages * Cfg::kStageBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + kEpiWarps * Cfg::kWarpStaging);
    const uint32_t full0 = ptx::smem_u32(bars), empty0 = full0 + 8 * Cfg::kStages;
    const uint32_t accfull0 = empty0 + 8 * Cfg::kStages, accempty0 = accfull0 + 16, stored0 = accempty0 + 16, drain = stored0 + 8 * (kUnitLag + 1);
    volatile uint32_t *tmem_holder = reinterpret_cast<volatile uint32_t *>(bars + 2 * Cfg::kStages + 5 + kUnitLag + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    volatile uint32_t *issued = tmem_holder + 2;
    const uint32_t ring = ptx::smem_u32(bars) + 256;                                            // this worker's units
    const uint32_t followed = ptx::smem_u32(const_cast<uint32_t *>(tmem_holder + 3)), loaded = followed + 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int worker = blockIdx.x / CG;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::kStages; ++s) {
            ptx::mbar_init(full0 + 8 * s, 1);
            ptx::mbar_init(empty0 + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(accfull0 + 8 * s, 1);
            ptx::mbar_init(accempty0 + 8 * s, kEpiWarps * CG);
        }
        for (int s = 0; s <= kUnitLag; ++s) ptx::mbar_init(stored0 + 8 * s, kEpiWarps);
        ptx::mbar_init(drain, 1);
        *abort_flag = 0;
        tmem_holder[3] = tmem_holder[4] = 0;
        for (int i = 0; i < 4 * kUnitRing; ++i) reinterpret_cast<volatile uint32_t *>(bars + 32)[i] = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async();
    }
    if (warp == 1) tmem_alloc_g<CG>(ptx::smem_u32(const_cast<uint32_t *>(tmem_holder)), Cfg::kTmemCols);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) cluster_sync();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_holder;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float grad_scale;
    const int n_units = muon_scale(p, grad_scale) ? p.n_units : 0;  // a bad scale leaves the step out
    int32_t taken = 0;  // of the worker's units, by this thread
    MuonUnit g{};
    auto next = [&] { return unit_next(g, ring, taken++, abort_flag, p.wait_limit_ns); };

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, asked = 0;
            bool ok = !(p.stall == 1 && worker == 0);
            const uint32_t full_base = CG == 2 ? map_to_rank(full0, 0) : full0;
            while (ok && next()) {
                const CUtensorMap *maps = p.maps + (int64_t)g.matrix * kMuonMaps;
                const int x = g.product / 3 & 1;
                // X X^T or X^T X, A A, and the polynomial times X from either side
                const CUtensorMap *map_a, *map_b;
                bool a_mn = false, b_mn = false;
                if (g.kind == 0) {
                    a_mn = b_mn = g.tall;
                    map_a = map_b = maps + (x ? kMapX1 : kMapX0) + (g.tall ? 1 : 0);
                } else if (g.kind == 1) {
                    map_a = map_b = maps + kMapGram;
                } else if (g.tall) {
                    map_a = maps + (x ? kMapX1 : kMapX0);
                    map_b = maps + kMapPoly;
                } else {
                    map_a = maps + kMapPoly;
                    map_b = maps + (x ? kMapX1N : kMapX0N);
                    b_mn = true;
                }
                const uint32_t bytes = CG * (g.same ? Cfg::kABytes : Cfg::kStageBytes);
                ptx::tensormap_acquire(map_a);
                ptx::tensormap_acquire(map_b);
                fence_proxy_async_all();  // what other SMs stored is read by tile loads
                const int32_t m0 = g.tm * Cfg::kTileRows + (int)rank * kGemmM, n0 = g.tn * BN + (int)rank * Cfg::kBRows;
                for (int kb = 0; kb < g.kblocks; ++kb) {
                    if (!ptx::mbar_wait_bounded(empty0 + 8 * stage, phase ^ 1u, abort_flag, p.wait_limit_ns)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = smem_base + stage * Cfg::kStageBytes, sb = sa + Cfg::kABytes;
                    if (rank == 0) ptx::mbar_arrive_expect_tx(full0 + 8 * stage, bytes);
                    const uint32_t bar = full_base + 8 * stage;
                    if (a_mn) {
#pragma unroll
                        for (int s = 0; s < kGemmM / 64; ++s) tma_load_g<CG>(sa + s * 8192, map_a, m0 + 64 * s, kb * kGemmK, bar);
                    } else {
                        tma_load_g<CG>(sa, map_a, kb * kGemmK, m0, bar);
                    }
                    if (g.same) {
                    } else if (b_mn) {
#pragma unroll
                        for (int s = 0; s < Cfg::kBRows / 64; ++s) tma_load_g<CG>(sb + s * 8192, map_b, n0 + 64 * s, kb * kGemmK, bar);
                    } else {
                        tma_load_g<CG>(sb, map_b, kb * kGemmK, n0, bar);
                    }
                    ++asked;
                    if (++stage == Cfg::kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (ok && rank == 0) units_raise(loaded, taken);
            }
            *issued = asked;
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc0 = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((kGemmM * CG) >> 4) << 24);
            uint32_t it = 0, acc = 0, acc_phase = 0;
            bool ok = true;
            const bool stop = p.stall == 2 && worker == 0;
            while (ok && next()) {
                const bool a_mn = g.kind == 0 && g.tall, b_mn = g.kind == 0 ? g.tall : g.kind == 2 && !g.tall;
                const uint32_t idesc = idesc0 | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16);
                const uint32_t step_a = a_mn ? 2048u >> 4 : 32u >> 4, step_b = b_mn ? 2048u >> 4 : 32u >> 4;
                const uint64_t base_a = a_mn ? make_desc_mn_sw128(0) : ptx::make_desc_k_sw128(0);
                const uint64_t base_b = b_mn ? make_desc_mn_sw128(0) : ptx::make_desc_k_sw128(0);
                if (!ptx::mbar_wait_bounded(accempty0 + 8 * acc, acc_phase ^ 1u, abort_flag, p.wait_limit_ns)) {
                    ok = false;
                    break;
                }
                ptx::tc_fence_after_sync();
                const int n = stop ? 1 : g.kblocks;
                for (int k = 0; k < n; ++k, ++it) {
                    const uint32_t s = it % Cfg::kStages;
                    if (!ptx::mbar_wait_bounded(full0 + 8 * s, (it / Cfg::kStages) & 1u, abort_flag, p.wait_limit_ns)) {
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t sa = smem_base + s * Cfg::kStageBytes, sb = g.same ? sa : sa + Cfg::kABytes;
                    mma_stage<BN, CG>(tmem + acc * BN, base_a | (sa >> 4), base_b | (sb >> 4), step_a, step_b, idesc, k == 0);
                    mma_commit_g<CG>(empty0 + 8 * s);
                }
                if (stop) ok = false;
                if (!ok) break;
                mma_commit_g<CG>(accfull0 + 8 * acc);
                acc ^= 1u;
                if (acc == 0) acc_phase ^= 1u;
            }
            if (!ok) {
                mma_commit_g<CG>(drain);
                const uint64_t t0 = ptx::globaltimer_ns();
                while (!ptx::mbar_try_wait(drain, 0))
                    if (ptx::globaltimer_ns() - t0 > p.wait_limit_ns) break;
            }
        }
        __syncwarp();
    } else if (warp < 2 + kEpiWarps) {
        const int e = warp - 2, quarter = warp & 3, strip = e >> 2;
        uint32_t acc = 0, acc_phase = 0;
        const uint32_t release0 = CG == 2 ? map_to_rank(accempty0, 0) : accempty0;
        Tile t;
        t.stage = reinterpret_cast<uint16_t *>(staging + e * Cfg::kWarpStaging);
        t.lane = lane;
        t.wide = 2;
        const uint32_t stage_at = ptx::smem_u32(t.stage);
        bool ok = true;
        while (ok && __all_sync(0xffffffffu, next())) {
            if (!__all_sync(0xffffffffu, units_wait(followed, taken - kUnitLag, abort_flag, p.wait_limit_ns))) break;
            const MuonMatrix q = p.matrices[g.matrix];  // (a copy: memory that may have changed would be read anew at every use)
            t.row0 = (int64_t)g.tm * Cfg::kTileRows + (int)rank * kGemmM + quarter * 32;
            t.rows = (int)min((g.kind == 2 ? q.rows : q.d) - t.row0, (int64_t)32);
            t.col0 = g.tn * BN + strip * Cfg::kColsPerWarp;
            t.cols = (int)min((g.kind == 2 ? q.cols : q.d) - t.col0, (int64_t)1 << 20);
            // all that the epilogue reads of the workspace is on its way while the products are computed
            const bool update = g.product + 1 == p.products;
            uint32_t ahead[Cfg::kPieces][16];
            uint32_t weights[2][16];
            auto fetch_update = [&] {
                if (t.rows <= 0 || t.cols <= 0) return;
                muon_fetch(ahead[0], q.lo, q.ldx, t);
                if (!NARROW || q.vector) with_type(q.param_type, [&](auto type) { muon_weights<decltype(type)>(weights, q, t); });
            };
            if (update) {
                fetch_update();
            } else if (g.kind != 0) {
                const uint16_t *from = g.kind == 1 ? q.gram : q.lo;
                const int64_t ld = g.kind == 1 ? q.ldd : q.ldx;
                Tile at = t;
#pragma unroll
                for (int c = 0; c < Cfg::kPieces; ++c) {
                    muon_fetch(ahead[c], from, ld, at);
                    at.col0 += kPiece;
                    at.cols -= kPiece;
                }
            }
            if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(accfull0 + 8 * acc, acc_phase, abort_flag, p.wait_limit_ns))) break;
            ptx::tc_fence_after_sync();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + strip * Cfg::kColsPerWarp;
            auto release = [&] {
                ptx::tc_fence_before_sync();
                if (lane == 0) {
                    if (CG == 2)
                        mbar_arrive_cluster(release0 + 8 * acc);
                    else
                        ptx::mbar_arrive(release0 + 8 * acc);
                }
            };
            auto add_rest = [](float (&v)[32], const uint32_t (&rest)[16]) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 l = unpack2<f16>(rest[i]);
                    v[2 * i] = fmaf(kNsA, l.x, v[2 * i]);
                    v[2 * i + 1] = fmaf(kNsA, l.y, v[2 * i + 1]);
                }
            };
            if (update) {
                const float keep = 1.0f - p.lr * q.wd, by = p.lr * q.scale * q.down;
                float *stage = reinterpret_cast<float *>(t.stage);
                with_type(q.param_type, [&](auto type) {
                    using P = decltype(type);
#pragma unroll 1
                    for (int c = 0; c < Cfg::kPieces; ++c) {
                        float v[32];
                        ptx::tmem_ld_32x32(src + c * kPiece, reinterpret_cast<uint32_t (&)[32]>(v));
                        ptx::tmem_ld_wait();
                        if (c == Cfg::kPieces - 1) release();
                        if (t.rows > 0 && t.cols > 0) {
                            add_rest(v, ahead[0]);
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                *reinterpret_cast<float4 *>(stage + lane * kUpdatePitch + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                            __syncwarp();
                            if (!NARROW || q.vector)
                                muon_update_wide<P>(q, weights, stage, keep, by, t);
                            else if (lane < t.cols)
                                muon_update_narrow<P>(static_cast<P *>(q.param) + t.row0 * q.cols + t.col0 + lane,
                                                      q.master ? q.master + t.row0 * q.cols + t.col0 + lane : nullptr, q.cols, stage + lane, keep, by, t.rows);
                        }
                        t.col0 += kPiece;
                        t.cols -= kPiece;
                        if (c + 1 < Cfg::kPieces) fetch_update();
                    }
                });
            } else if (g.kind == 2) {
                // X and its rest, 64 columns at a time
#pragma unroll
                for (int c = 0; c < Cfg::kPieces; c += 2) {
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float v[32];
                        ptx::tmem_ld_32x32(src + (c + h) * kPiece, reinterpret_cast<uint32_t (&)[32]>(v));
                        ptx::tmem_ld_wait();
                        if (c + h == Cfg::kPieces - 1) release();
                        add_rest(v, ahead[c + h]);
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            hi[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
                            const float2 f = unpack2<f16>(hi[i]);
                            lo[i] = pack2<f16>(v[2 * i] - f.x, v[2 * i + 1] - f.y);
                        }
                        stage_rows<64>(stage_at, 4 * h, hi, lane);
                        stage_rows<64>(stage_at + 4096, 4 * h, lo, lane);
                    }
                    __syncwarp();
                    const int64_t to = t.row0 * q.ldx + t.col0;
                    const int cols = min((int)q.ldx - t.col0, 2 * kPiece);
                    store_staged<64>(stage_at, (g.product / 3 & 1 ? q.x[0] : q.x[1]) + to, q.ldx, t.rows, cols, lane);
                    store_staged<64>(stage_at + 4096, q.lo + to, q.ldx, t.rows, cols, lane);
                    t.col0 += 2 * kPiece;
                }
            } else {
                // A, or the polynomial: the pieces on and above the diagonal and the mirror images of the latter
                uint16_t *const to = g.kind == 0 ? q.gram : q.poly;
                const float down = q.down * q.down;
#pragma unroll
                for (int c = 0; c < Cfg::kPieces; ++c) {
                    float v[32];
                    ptx::tmem_ld_32x32(src + c * kPiece, reinterpret_cast<uint32_t (&)[32]>(v));
                    ptx::tmem_ld_wait();
                    if (c == Cfg::kPieces - 1) release();
                    if (t.rows > 0 && t.cols > 0 && t.row0 <= t.col0) {
                        if (g.kind == 0) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] *= down;
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 h = unpack2<f16>(ahead[c][i]);
                                v[2 * i] = fmaf(kNsC, v[2 * i], kNsB * h.x);
                                v[2 * i + 1] = fmaf(kNsC, v[2 * i + 1], kNsB * h.y);
                            }
                            if (t.row0 == t.col0) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] += lane == i ? kNsA : 0.0f;
                            }
                        }
                        uint32_t r[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
                        const uint32_t at = stage_at + (c & 1) * 4096;
                        __syncwarp();
                        stage_rows<32>(at, 0, r, lane);
                        if (t.row0 < t.col0) stage_mirror(at + 2048, r, lane);
                        __syncwarp();
                        store_staged<32>(at, to + t.row0 * q.ldd + t.col0, q.ldd, t.rows, kPiece, lane);
                        if (t.row0 < t.col0) store_staged<32>(at + 2048, to + t.col0 * (int64_t)q.ldd + t.row0, q.ldd, t.cols, kPiece, lane);
                    }
                    t.col0 += kPiece;
                    t.cols -= kPiece;
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(stored0 + 8 * ((taken - 1) % (kUnitLag + 1)));
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        }
    } else if (warp == 2 + kEpiWarps + 1) {
        if (lane == 0 && rank == 0) {
            // The units are taken from the head of the list in turn.  Where there are plenty, each while the one before is being loaded;
            // else not before that, so that none waits here which another worker could begin.
            const uint32_t ring1 = CG == 2 ? map_to_rank(ring, 1) : 0;
            while (p.stall != 1 || worker != 0) {
                if (!units_wait(loaded, taken - p.early, abort_flag, p.wait_limit_ns)) break;
                const int32_t u = atomicAdd(p.ticket, 1);
                const int4 q = u < n_units ? p.units[u] : make_int4(kNoMoreUnits, 0, 0, 0);
                if (q.x != kNoMoreUnits) {
                    g = muon_unit(q);
                    if (!eg_check(g.matrix < p.n_matrices && g.product < p.products, p.status, kCheckMuonUnit, g.matrix)) break;
                    const int state = muon_wait(p.done + g.matrix, g.need, abort_flag, p.wait_limit_ns);
                    if (state == 0) break;
                    if (state < 0) continue;
                }
                unit_publish<CG>(ring, ring1, q, taken);
                ++taken;
                if (q.x == kNoMoreUnits) break;
            }
        }
        __syncwarp();
    } else if (lane == 0) {
        // When all of the epilogue's warps have stored their part of a tile, it is made known.
        while (next()) {
            units_raise(followed, taken);
            const int32_t n = taken - 1;
            if (!ptx::mbar_wait_bounded(stored0 + 8 * (n % (kUnitLag + 1)), (uint32_t)(n / (kUnitLag + 1)) & 1u, abort_flag, p.wait_limit_ns)) break;
            if (g.product + 1 == p.products) continue;  // the update, for which nothing waits
            fence_proxy_async_all();
            __threadfence();
            atomicAdd(p.done + g.matrix, 1);
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {
        // as in gemm_kernel
        const uint64_t t0 = ptx::globaltimer_ns();
        if (rank == 0) {
            const uint32_t asked = *issued;
            for (uint32_t k = 1; k <= min(asked, (uint32_t)Cfg::kStages); ++k) {
                const uint32_t idx = asked - k, s = idx % Cfg::kStages, ph = (idx / Cfg::kStages) & 1u;
                while (!ptx::mbar_try_wait(full0 + 8 * s, ph))
                    if (ptx::globaltimer_ns() - t0 > p.wait_limit_ns) break;
            }
        } else {
            while (ptx::globaltimer_ns() - t0 < 1000000ull) {
            }
        }
        atomicMax(p.status, 6);
    }
    if (CG == 2) cluster_sync();
    ptx::tc_fence_after_sync();
    if (warp == 1) tmem_free_g<CG>(tmem, Cfg::kTmemCols);
}

// ---------------------------------------------------------------- small matrices
// The whole step of a matrix of at most 128 by 768 in one thread block: X stays in shared memory, as the products' operand from either
// side (its 64-column panels are A X^T's with the columns consecutive and P X's with them as the other axis), and only what its
// rounding leaves goes by way of L2.  54 convolutions of 16 to 64 channels: 58 us, 100 through the list of units, where each of the 15
// products waits for the one before it to be stored, seen and loaded.  Of the 58, 10 go into the first 64 x 576 X and 6 into its
// weights (0.7 and 0.4 MB through one SM at the 60 to 70 bytes a nanosecond that these loads get), 7.3 into each of the five steps: 1.1 of waiting for
// A, 0.9 for A A, 4.9 for three chunks, whose products and values and the next A's part of them run beside each other (8.6 before).
constexpr int kSmallSide = 128, kSmallPanels = 12;
constexpr int kSmallThreads = 512, kSmallStrips = kSmallThreads / 128, kPanelBytes = kSmallSide * 128;
constexpr int kChunk = 3;                                       // panels whose new values are computed at a time
constexpr int kSquareAt = 2 * kChunk * 64;                      // where A and A A are in tensor memory, beside two chunks
constexpr int kSmallSmem = 1024 + (kSmallPanels + 2) * kPanelBytes + 256;
static_assert(kSmallSmem <= 227 * 1024 && kSquareAt + kSmallSide <= 512, "shared and tensor memory of a CTA");

// Place of a value in a panel: rows of 64 values, 128 bytes, swizzled as the tensor cores take them.
__device__ __forceinline__ uint32_t panel_place(uint32_t row, uint32_t col) {
    return (col >> 6) * kPanelBytes + row * 128 + (((col >> 3 & 7) ^ (row & 7)) << 4) + (col & 7) * 2;
}
// Place of a value of X's rest in the workspace: eights of columns, a row per lane.
__device__ __forceinline__ int32_t rest_place(int32_t row, int32_t col) { return ((col >> 3) * kSmallSide + row) * 8 + (col & 7); }
// 32 values of a row from a multiple of 32 columns on.
__device__ __forceinline__ void panel_store(uint32_t base, uint32_t row, uint32_t col, const uint32_t (&r)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + panel_place(row, col + 8 * i)), "r"(r[4 * i]), "r"(r[4 * i + 1]),
                     "r"(r[4 * i + 2]), "r"(r[4 * i + 3])
                     : "memory");
}

// A thread's eights of a matrix, kSmallGroup of them loaded before the first is used: a block alone on its SM has no other loads to wait
// beside.
constexpr int kSmallGroup = 3;

// Momentum, |t|, and X in the panels with its rest in `lo`.
template <bool VECTOR, typename G>
__device__ __forceinline__ void small_begin(const MuonParams &p, const MuonMatrix &t, const G *grad, float grad_scale, uint32_t base, double *part) {
    constexpr int S = VECTOR ? 1 : kSmallThreads;  // between a thread's eight values
    constexpr int kStep = 8 * kSmallThreads;
    const int32_t cols = (int32_t)t.cols, n = (int32_t)(t.rows * t.cols), first = threadIdx.x * (VECTOR ? 8 : 1);
    double sum = 0.0;
#pragma unroll 1
    for (int32_t e0 = first; e0 < n; e0 += kSmallGroup * kStep) {
        float g[kSmallGroup][8], m[kSmallGroup][8];
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
            muon_read<VECTOR, S>(g[j], grad, e, n);
            muon_read<VECTOR, S>(m[j], t.m, e, n);
        }
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gi = g[j][i] * grad_scale;
                m[j][i] = fmaf(p.beta, m[j][i], p.rest * gi);
                const float v = p.nesterov ? fmaf(p.beta, m[j][i], p.rest * gi) : m[j][i];
                if (VECTOR || e + i * S < n) sum = fma((double)v, (double)v, sum);
            }
            if (VECTOR) {
                store8(t.m + e, m[j]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e + i * S < n) t.m[e + i * S] = m[j][i];
            }
        }
    }
    const float inv = (float)((double)t.up / fmax(sqrt(block_sum<kSmallThreads>(sum, part)), (double)p.eps));
#pragma unroll 1
    for (int32_t e0 = first; e0 < n; e0 += kSmallGroup * kStep) {  // (its own values of m again)
        float g[kSmallGroup][8], v[kSmallGroup][8];
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
            muon_read<VECTOR, S>(v[j], t.m, e, n);
            if (p.nesterov) muon_read<VECTOR, S>(g[j], grad, e, n);
        }
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
            if (p.nesterov) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = fmaf(p.beta, v[j][i], p.rest * (g[j][i] * grad_scale));
            }
            uint32_t h[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = pack2<f16>(v[j][2 * i] * inv, v[j][2 * i + 1] * inv);
                const float2 f = unpack2<f16>(h[i]);
                l[i] = pack2<f16>(v[j][2 * i] * inv - f.x, v[j][2 * i + 1] * inv - f.y);
            }
            const int32_t r = e / cols, c = e - r * cols;
            if (VECTOR && !t.tall) {  // eight values of a row, which is one of X
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + panel_place(r, c)), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
                *reinterpret_cast<uint4 *>(t.lo + rest_place(r, c)) = make_uint4(l[0], l[1], l[2], l[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t at = e + i * S;
                    if (at >= n) break;
                    const int32_t ri = VECTOR ? r : at / cols, ci = VECTOR ? c + i : at - ri * cols, row = t.tall ? ci : ri, col = t.tall ? ri : ci;
                    const uint16_t hi = (uint16_t)(h[i >> 1] >> (i & 1) * 16), lo = (uint16_t)(l[i >> 1] >> (i & 1) * 16);
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(base + panel_place(row, col)), "h"(hi) : "memory");
                    t.lo[rest_place(row, col)] = lo;
                }
            }
        }
    }
}

// p = p keep - step X, in the order of the weights.
template <typename T, bool VECTOR>
__device__ __forceinline__ void small_end(const MuonParams &p, const MuonMatrix &t, uint32_t base) {
    constexpr int S = VECTOR ? 1 : kSmallThreads, kStep = 8 * kSmallThreads;
    const int32_t cols = (int32_t)t.cols, n = (int32_t)(t.rows * t.cols);
    const float keep = 1.0f - p.lr * t.wd, by = p.lr * t.scale * t.down;
    T *param = static_cast<T *>(t.param);
#pragma unroll 1
    for (int32_t e0 = threadIdx.x * (VECTOR ? 8 : 1); e0 < n; e0 += kSmallGroup * kStep) {
        float w[kSmallGroup][8];
        uint4 rest[kSmallGroup];
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
            if (t.master)
                muon_read<VECTOR, S>(w[j], t.master, e, n);
            else
                muon_read<VECTOR, S>(w[j], param, e, n);
            if (VECTOR && !t.tall) {
                const int32_t r = e / cols;
                rest[j] = *reinterpret_cast<const uint4 *>(t.lo + rest_place(r, e - r * cols));
            }
        }
#pragma unroll
        for (int j = 0; j < kSmallGroup; ++j) {
            const int32_t e = e0 + j * kStep;
            if (e >= n) break;
            const int32_t r = e / cols, c = e - r * cols;
            float x[8];
            if (VECTOR && !t.tall) {
                uint32_t h[4];
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
                             : "r"(base + panel_place(r, c))
                             : "memory");
                const uint32_t l[4] = {rest[j].x, rest[j].y, rest[j].z, rest[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack2<f16>(h[i]), g = unpack2<f16>(l[i]);
                    x[2 * i] = f.x + g.x, x[2 * i + 1] = f.y + g.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t at = min(e + i * S, n - 1);
                    const int32_t ri = VECTOR ? r : at / cols, ci = VECTOR ? c + i : at - ri * cols, row = t.tall ? ci : ri, col = t.tall ? ri : ci;
                    uint16_t h;
                    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(h) : "r"(base + panel_place(row, col)) : "memory");
                    x[i] = __half2float(__ushort_as_half(h)) + __half2float(__ushort_as_half(t.lo[rest_place(row, col)]));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) w[j][i] = fmaf(w[j][i], keep, -by * x[i]);
            if (VECTOR) {
                store8(param + e, w[j]);
                if (t.master) store8(t.master + e, w[j]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e + i * S < n) {
                        param[e + i * S] = from_f32<T>(w[j][i]);
                        if (t.master) t.master[e + i * S] = w[j][i];
                    }
            }
        }
    }
}

__global__ void __launch_bounds__(kSmallThreads, 1) muon_small_kernel(const __grid_constant__ MuonParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ double part[kSmallThreads / 32];
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_word;
    __shared__ alignas(8) uint64_t bars[4];  // a chunk of either parity, A or A A, the end of what was begun
    const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, poly = base + kSmallPanels * kPanelBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3, strip = warp >> 2;
    // issues the products: of the warp that has least to do beside (none up to 96 rows), since it stands still while the queue is full
    const bool leader = threadIdx.x == kSmallThreads - 32;
    volatile int *abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) ptx::mbar_init(ptx::smem_u32(bars + i), 1);
        abort_word = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async();
    }
    if (warp == 0) tmem_alloc_g<1>(ptx::smem_u32(&tmem_holder), 512);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = tmem_holder;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float grad_scale;
    const bool fine = muon_scale(p, grad_scale) && eg_check(p.first_small + (int)blockIdx.x < p.n_matrices, p.status, kCheckMuonUnit, blockIdx.x);
    const MuonMatrix t = p.matrices[fine ? p.first_small + blockIdx.x : 0];
    if (fine && !muon_skips(p, t)) {
        const int32_t d = t.d, len = (int32_t)max(t.rows, t.cols);
        const int32_t panels = (len + 63) / 64;
        const void *grad = p.grads[t.index];
        // the panels' zeros (the rest holds anything behind a row's end, where it is not looked at)
        for (int i = threadIdx.x; i < panels * kPanelBytes / 16; i += kSmallThreads)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + i * 16), "r"(0) : "memory");
        const bool vector = muon_vector(p, t);
        __syncthreads();
        with_type(t.grad_type, [&](auto type) {
            const auto *g = static_cast<const decltype(type) *>(grad);
            if (vector)
                small_begin<true>(p, t, g, grad_scale, base, part);
            else
                small_begin<false>(p, t, g, grad_scale, base, part);
        });
        const int steps = p.products / 3;
        uint32_t phases = 0;
        bool ok = true;
        const uint32_t row = quarter * 32 + lane;
        const uint32_t tmem_row = tmem + ((uint32_t)(quarter * 32) << 16);
        auto idesc = [](int cols, bool b_mn) { return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(cols >> 3) << 17) | ((uint32_t)(kSmallSide >> 4) << 24); };
        // everything that has been stored in shared memory, and read from tensor memory, comes before the products
        // (where a wait ran out, which all learn of here, what was stored since then is not used)
        auto meet = [&] {
            ptx::fence_proxy_async();
            ptx::tc_fence_before_sync();
            ok = __syncthreads_and(ok);
            ptx::tc_fence_after_sync();
            return ok;
        };
        // A warp's pieces of a chunk (two at most), and what X's rounding left of them.  A thread reads back what it wrote itself; the
        // loads are under way from the chunk or the step before.
        uint32_t lo[2][16];
        auto has_piece = [&](int c, int k) { return strip + k * kSmallStrips < min(kChunk, panels - kChunk * c) * 2 && (int)row < d; };
        auto rest_at = [&](int c, int k) { return t.lo + rest_place(row, c * kChunk * 64 + (strip + k * kSmallStrips) * kPiece); };
        auto fetch_rest = [&](int c, int k) {
            if (!has_piece(c, k)) return;
            const uint4 *rest = reinterpret_cast<const uint4 *>(rest_at(c, k));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 q = rest[i * kSmallSide];
                lo[k][4 * i] = q.x, lo[k][4 * i + 1] = q.y, lo[k][4 * i + 2] = q.z, lo[k][4 * i + 3] = q.w;
            }
        };
        auto store_rest = [&](int c, int k) {
            if (!has_piece(c, k)) return;
            uint4 *rest = reinterpret_cast<uint4 *>(rest_at(c, k));
#pragma unroll
            for (int i = 0; i < 4; ++i) rest[i * kSmallSide] = make_uint4(lo[k][4 * i], lo[k][4 * i + 1], lo[k][4 * i + 2], lo[k][4 * i + 3]);
        };
        auto wait = [&](int bar) {
            ok = ok && ptx::mbar_wait_bounded(ptx::smem_u32(bars + bar), phases >> bar & 1u, abort_flag, p.wait_limit_ns);
            phases ^= 1u << bar;
            ptx::tc_fence_after_sync();
        };
        const int ksteps = (d + 15) / 16;       // of a sum over the shorter side
        const int side = (d + 31) / 32 * 32;    // rows and columns of A that are looked at (tensor memory's others hold anything)
        const bool mine = quarter * 32 < side && strip * 32 < side;
        // a product's steps of 16, four with the same start addresses at a time
        auto over = [](int n, auto go) {
#pragma unroll 1
            for (int k = 0; k < n; k += 4)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k + i < n) go(k, i);
        };
        // the product of n steps of an operand with itself, added to what is there or not
        auto square = [&](uint32_t at, int n, bool more) {
            const uint64_t x0 = ptx::make_desc_k_sw128(at);
            over(n, [&](int k, int i) {
                const uint64_t x = x0 + (uint32_t)(k >> 2) * (kPanelBytes >> 4) + i * 2;
                mma_g<1>(tmem + kSquareAt, x, x, idesc(side, false), more || k + i > 0);
            });
        };
        // P X for the panels of chunk c into the accumulator of its parity, and X X^T's part of it
        const int chunks = (panels + kChunk - 1) / kChunk;
        auto issue_chunk = [&](int c) {
            const int wide = min(kChunk, panels - kChunk * c) * 64;
            const uint64_t mn = (uint64_t)(kPanelBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
            const uint64_t p0 = ptx::make_desc_k_sw128(poly), x0 = mn | (base + kChunk * c * kPanelBytes) >> 4;
            over(ksteps, [&](int k, int i) {
                mma_g<1>(tmem + (c & 1) * kChunk * 64, p0 + (uint32_t)(k >> 2) * (kPanelBytes >> 4) + i * 2, x0 + (uint32_t)(k + i) * (2048 >> 4),
                         idesc(wide, true), k + i > 0);
            });
            mma_commit_g<1>(ptx::smem_u32(bars + (c & 1)));
        };
        auto square_chunk = [&](int c) { square(base + kChunk * c * kPanelBytes, min(kChunk, panels - kChunk * c) * 4, c > 0); };
        meet();
        // A = X X^T
        if (leader && p.stall == 0) {
            square(base, panels * 4, false);
            mma_commit_g<1>(ptx::smem_u32(bars + 2));
        }
        fetch_rest(0, 0);
        fetch_rest(0, 1);
#pragma unroll 1
        for (int step = 0; step < steps && ok; ++step) {
            wait(2);
            uint32_t a[16];
            const float down = t.down * t.down;
            if (mine) {
                float v[32];
                ptx::tmem_ld_32x32(tmem_row + kSquareAt + strip * 32, reinterpret_cast<uint32_t (&)[32]>(v));
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) a[i] = pack2<f16>(v[2 * i] * down, v[2 * i + 1] * down);
                panel_store(poly, row, strip * 32, a);
            }
            if (!meet()) break;
            // A A, and P over A
            if (leader) {
                square(poly, ksteps, false);
                mma_commit_g<1>(ptx::smem_u32(bars + 2));
            }
            wait(2);
            if (mine) {
                float v[32];
                ptx::tmem_ld_32x32(tmem_row + kSquareAt + strip * 32, reinterpret_cast<uint32_t (&)[32]>(v));
                ptx::tmem_ld_wait();
                const int diagonal = (int)row < d ? (int)row - strip * 32 : -1;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 f = unpack2<f16>(a[i]);
                    v[2 * i] = fmaf(kNsC, v[2 * i], kNsB * f.x) + (diagonal == 2 * i ? kNsA : 0.0f);
                    v[2 * i + 1] = fmaf(kNsC, v[2 * i + 1], kNsB * f.y) + (diagonal == 2 * i + 1 ? kNsA : 0.0f);
                }
                uint32_t r[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) r[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
                panel_store(poly, row, strip * 32, r);
            }
            if (!meet()) break;
            // X = P X, a chunk at a time: its products run beside the values of the chunk before, and so does the next A's part of that
            const bool again = step + 1 < steps;
            if (leader) {
                issue_chunk(0);
                if (chunks > 1) issue_chunk(1);
            }
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                wait(c & 1);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = strip + k * kSmallStrips;
                    if (at >= min(kChunk, panels - kChunk * c) * 2 || quarter * 32 >= side) continue;
                    const int32_t col = c * kChunk * 64 + at * kPiece;
                    float v[32];
                    ptx::tmem_ld_32x32(tmem_row + (c & 1) * kChunk * 64 + at * kPiece, reinterpret_cast<uint32_t (&)[32]>(v));
                    ptx::tmem_ld_wait();
                    if ((int)row < d) {  // (whole rows of zeros stay as they are)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 f = unpack2<f16>(lo[k][i]);
                            v[2 * i] = col + 2 * i < len ? fmaf(kNsA, f.x, v[2 * i]) : 0.0f;
                            v[2 * i + 1] = col + 2 * i + 1 < len ? fmaf(kNsA, f.y, v[2 * i + 1]) : 0.0f;
                        }
                        uint32_t hi[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            hi[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
                            const float2 f = unpack2<f16>(hi[i]);
                            lo[k][i] = pack2<f16>(v[2 * i] - f.x, v[2 * i + 1] - f.y);
                        }
                        panel_store(base, row, col, hi);
                    }
                }
                if (!meet()) break;  // (the accumulator of this chunk is free for the chunk after the next)
                if (leader) {
                    if (c + 2 < chunks) issue_chunk(c + 2);
                    if (again) square_chunk(c);
                    if (again && c + 1 == chunks) mma_commit_g<1>(ptx::smem_u32(bars + 2));
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    store_rest(c, k);
                    fetch_rest(c + 1 < chunks ? c + 1 : 0, k);
                }
            }
        }
        // (the last X's rest is read by others)
        __syncthreads();
        if (ok)
            with_type(t.param_type, [&](auto type) {
                if (t.vector)
                    small_end<decltype(type), true>(p, t, base);
                else
                    small_end<decltype(type), false>(p, t, base);
            });
        if (!ok && leader) {
            // gave up: no product of ours may still read shared memory when the block leaves
            mma_commit_g<1>(ptx::smem_u32(bars + 3));
            const uint64_t t0 = ptx::globaltimer_ns();
            while (!ptx::mbar_try_wait(ptx::smem_u32(bars + 3), 0))
                if (ptx::globaltimer_ns() - t0 > p.wait_limit_ns) break;
            atomicMax(p.status, 6);
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    if (warp == 0) tmem_free_g<1>(tmem, 512);
}

}  // namespace ops
}  // namespace egeria
