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
// Operands are f16, sums 32 bits.  All values are below 2 in size, where f16 has three bits more than bf16.  A and the
// polynomial are rounded once each.  X is kept as two f16 values, the second what the first leaves (22 bits): the products take the
// first alone, but where X is added to itself both count.  A rounding of X there would lie across its null space too, which no
// product damps and every step multiplies by a: a 1024 x 1024 matrix of rank 64 is off by 5.8e-4 (2-norm of the difference
// over that of the result, from the formula in 64 bits), with X in one f16 value by 2.4e-2, in one bf16 value by 0.19; a matrix of
// independent normal values by 1.3e-3, 1.2e-3 and 9.3e-3.  X is held times a power of two, so that its values stay off f16's
// lower end.
//
// All products of all matrices are one launch: a list of units (a tile of one of the 3 `steps` products of one matrix), dealt round
// the workers (CTAs, or pairs of them).  A unit waits until the units of its matrix's product before it are done, which a
// counter per matrix says; the list has several matrices' tiles of a product side by side, so that as a rule it is long done.
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
    const int4 *units;               // matrix, tm | tn << 16, product | k blocks << 8, count that the matrix's counter has to reach
    const int2 *pieces;              // matrix, piece
    const void *const *grads;
    int32_t *done;                   // per matrix
    int32_t *status;
    const float *grad_scale;
    const uint8_t *frozen;
    float lr, beta, rest, eps;
    int32_t nesterov, n_units, n_pieces, n_matrices, products;
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
// Eight gradients from value e of a matrix on; those behind n count as 0.
template <bool VECTOR>
__device__ __forceinline__ void muon_grads(float (&g)[8], const void *grad, int type, int64_t e, int64_t n) {
    auto go = [&](auto *p) {
        using T = typename std::remove_const<typename std::remove_reference<decltype(*p)>::type>::type;
        if (VECTOR) {
            Raw8<T> r;
            load8(r, p + e);
            unpack8(g, r);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = e + i < n ? to_f32(p[e + i]) : 0.0f;
        }
    };
    if (type == EGERIA_F32)
        go(static_cast<const float *>(grad));
    else if (type == EGERIA_BF16)
        go(static_cast<const bf16 *>(grad));
    else
        go(static_cast<const f16 *>(grad));
}
template <bool VECTOR>
__device__ __forceinline__ void muon_moments(float (&m)[8], const float *p, int64_t e, int64_t n) {
    if (VECTOR) {
        Raw8<float> r;
        load8(r, p + e);
        unpack8(m, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = e + i < n ? p[e + i] : 0.0f;
    }
}
__device__ __forceinline__ double block_sum(double v, double *part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kMuonThreads / 32; ++w) v += part[w];
    return v;
}

// The momentum, and the sum of t^2 of each piece (in 64 bits: neither tiny nor huge gradients leave the range).
template <bool VECTOR>
__device__ __forceinline__ double muon_momentum_piece(const MuonParams &p, const MuonMatrix &t, int64_t e0, float scale) {
    const int64_t n = t.rows * t.cols, end = min(n, e0 + kMuonPiece);
    const void *grad = p.grads[t.index];
    double sum = 0.0;
    for (int64_t e = e0 + threadIdx.x * 8; e < end; e += kMuonThreads * 8) {
        float g[8], m[8];
        muon_grads<VECTOR>(g, grad, t.grad_type, e, n);
        muon_moments<VECTOR>(m, t.m, e, n);
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
                if (e + i < n) t.m[e + i] = m[i];
        }
    }
    return sum;
}
__global__ void __launch_bounds__(kMuonThreads) muon_momentum_kernel(const MuonParams p) {
    __shared__ double part[kMuonThreads / 32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < p.n_matrices; i += kMuonThreads) p.done[i] = 0;
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
    for (int64_t e = e0 + threadIdx.x * 8; e < end; e += kMuonThreads * 8) {
        float g[8], v[8];
        muon_moments<VECTOR>(v, t.m, e, n);
        if (p.nesterov) {
            muon_grads<VECTOR>(g, grad, t.grad_type, e, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(p.beta, v[i], p.rest * (g[i] * scale));
        }
        uint32_t at = c0 + (uint32_t)(e - e0), row = at / cols, col = at - row * cols;
        uint16_t *x = t.x[0] + (r0 + row) * t.ldx + col, *lo = t.lo + (r0 + row) * t.ldx + col;
        if (VECTOR) {  // whole eights of a row
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
                if (e + i >= n) break;
                f16 h, l;
                muon_split(v[i] * inv, h, l);
                *x++ = __half_as_ushort(h);
                *lo++ = __half_as_ushort(l);
                if (++col == cols) {
                    col = 0;
                    x += t.ldx - cols;
                    lo += t.ldx - cols;
                }
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
// different SMs within one launch: past L1.
__device__ __forceinline__ void muon_fetch(uint32_t (&r)[16], const uint16_t *base, int64_t ld, const Tile &t) {
    if (t.lane < t.rows) {
        const uint4 *p = reinterpret_cast<const uint4 *>(base + (t.row0 + t.lane) * ld + t.col0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = __ldcg(p + i);
            r[4 * i] = q.x, r[4 * i + 1] = q.y, r[4 * i + 2] = q.z, r[4 * i + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = 0u;
    }
}
__device__ __forceinline__ void muon_store(uint16_t *base, int64_t ld, const uint32_t (&r)[16], const Tile &t) {
    if (t.lane < t.rows) {
        uint16_t *p = base + (t.row0 + t.lane) * ld + t.col0;
        ptx::st_global_v8(reinterpret_cast<float *>(p), r);
        ptx::st_global_v8(reinterpret_cast<float *>(p + 16), r + 8);
    }
}
// A piece of a symmetric matrix and its mirror image.  Pieces below the diagonal are left to their images.
__device__ __forceinline__ void muon_store_symmetric(uint16_t *base, int64_t ld, const float (&v)[32], const Tile &t) {
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
    muon_store(base, ld, r, t);
    if (t.row0 == t.col0) return;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) reinterpret_cast<uint32_t *>(t.stage)[t.lane * (kStagePitch / 2) + i] = r[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i)
        r[i] = (uint32_t)t.stage[(2 * i) * kStagePitch + t.lane] | (uint32_t)t.stage[(2 * i + 1) * kStagePitch + t.lane] << 16;
    Tile s = t;
    s.row0 = t.col0;
    s.rows = t.cols;
    s.col0 = (int32_t)t.row0;
    muon_store(base, ld, r, s);
}

// p = p keep - step X of a piece, x: X's values.
template <typename T>
__device__ __forceinline__ void muon_update_values(T *param, float *master, int64_t at, float x, float keep, float step) {
    const float v = fmaf(master ? master[at] : to_f32(param[at]), keep, -step * x);
    param[at] = from_f32<T>(v);
    if (master) master[at] = v;
}
template <typename T>
__device__ __forceinline__ void muon_update(const MuonMatrix &q, float (&x)[32], float keep, float step, const Tile &t) {
    T *param = static_cast<T *>(q.param);
    if (q.vector && t.cols >= kPiece) {
        if (t.lane < t.rows) {
            const int64_t at = (t.row0 + t.lane) * q.cols + t.col0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[8];
                if (q.master) {
                    Raw8<float> r;
                    load8(r, q.master + at + 8 * i);
                    unpack8(v, r);
                } else {
                    Raw8<T> r;
                    load8(r, param + at + 8 * i);
                    unpack8(v, r);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = fmaf(v[k], keep, -step * x[8 * i + k]);
                store8(param + at + 8 * i, v);
                if (q.master) store8(q.master + at + 8 * i, v);
            }
        }
        return;
    }
    // row by row, with lane = column, sixteen columns of the piece at a time through shared memory
    const int rows = min(t.rows, 32), c = t.lane & 15;
    float *stage = reinterpret_cast<float *>(t.stage);  // [32][17]
    for (int half = 0; half < 2; ++half) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) stage[t.lane * 17 + i] = half ? x[16 + i] : x[i];
        __syncwarp();
        if (half * 16 + c < t.cols)
            for (int k = t.lane >> 4; k < rows; k += 2)
                muon_update_values(param, q.master, (t.row0 + k) * q.cols + t.col0 + half * 16 + c, stage[k * 17 + c], keep, step);
    }
}

__device__ __forceinline__ int32_t load_acquire(const int32_t *p) {
    int32_t v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Until the counter has come that far, but not for ever.
__device__ __forceinline__ bool muon_wait(const int32_t *done, int32_t need, volatile int *abort_flag, uint64_t limit_ns) {
    if (load_acquire(done) >= need) return true;
    const uint64_t t0 = ptx::globaltimer_ns();
    while (load_acquire(done) < need) {
        if (*abort_flag) return false;
        if (ptx::globaltimer_ns() - t0 > limit_ns) {
            *abort_flag = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

struct MuonUnit {
    int32_t matrix, tm, tn, product, kblocks, need;
};
__device__ __forceinline__ MuonUnit muon_unit(const MuonParams &p, int u) {
    const int4 q = p.units[u];
    return MuonUnit{q.x, q.y & 0xffff, q.y >> 16 & 0xffff, q.z & 0xff, (int32_t)((uint32_t)q.z >> 8), q.w};
}

template <int BN, int CG>
__global__ void __launch_bounds__(GemmCfg<BN, CG, 1>::kThreads, 1) muon_products_kernel(const __grid_constant__ MuonParams p) {
    using Cfg = GemmCfg<BN, CG, 1>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    uint16_t *staging = reinterpret_cast<uint16_t *>(smem + Cfg::kStages * Cfg::kStageBytes);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Cfg::kStages * Cfg::kStageBytes + Cfg::kStaging);
    const uint32_t full0 = ptx::smem_u32(bars), empty0 = full0 + 8 * Cfg::kStages;
    const uint32_t accfull0 = empty0 + 8 * Cfg::kStages, accempty0 = accfull0 + 16, drain = accempty0 + 16;
    volatile uint32_t *tmem_holder = reinterpret_cast<volatile uint32_t *>(bars + 2 * Cfg::kStages + 5);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    volatile uint32_t *issued = tmem_holder + 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::kStages; ++s) {
            ptx::mbar_init(full0 + 8 * s, 1);
            ptx::mbar_init(empty0 + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(accfull0 + 8 * s, 1);
            ptx::mbar_init(accempty0 + 8 * s, kEpiWarps * CG);
        }
        ptx::mbar_init(drain, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async();
    }
    if (warp == 1) tmem_alloc_g<CG>(ptx::smem_u32(const_cast<uint32_t *>(tmem_holder)), Cfg::kTmemCols);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) cluster_sync();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_holder;
    float grad_scale;
    const int n_units = muon_scale(p, grad_scale) ? p.n_units : 0;  // a bad scale leaves the step out
    auto left_out = [&](const MuonUnit &g) {
        return !eg_check(g.matrix >= 0 && g.matrix < p.n_matrices, p.status, kCheckMuonUnit, g.matrix) || muon_skips(p, p.matrices[g.matrix]);
    };

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, asked = 0;
            bool ok = !(p.stall == 1 && worker == 0);
            const uint32_t full_base = CG == 2 ? map_to_rank(full0, 0) : full0;
            for (int u = worker; ok && u < n_units; u += workers) {
                const MuonUnit g = muon_unit(p, u);
                if (left_out(g)) continue;
                const MuonMatrix &q = p.matrices[g.matrix];
                const CUtensorMap *maps = p.maps + (int64_t)g.matrix * kMuonMaps;
                const int kind = g.product % 3, x = g.product / 3 & 1;
                // A X^T and X^T X, A A, and the polynomial times X from either side
                const CUtensorMap *map_a, *map_b;
                bool a_mn = false, b_mn = false;
                if (kind == 0) {
                    a_mn = b_mn = q.tall;
                    map_a = map_b = maps + (x ? kMapX1 : kMapX0) + (q.tall ? 1 : 0);
                } else if (kind == 1) {
                    map_a = map_b = maps + kMapGram;
                } else if (q.tall) {
                    map_a = maps + (x ? kMapX1 : kMapX0);
                    map_b = maps + kMapPoly;
                } else {
                    map_a = maps + kMapPoly;
                    map_b = maps + (x ? kMapX1N : kMapX0N);
                    b_mn = true;
                }
                ptx::tensormap_acquire(map_a);
                ptx::tensormap_acquire(map_b);
                if (!muon_wait(p.done + g.matrix, g.need, abort_flag, p.wait_limit_ns)) break;
                fence_proxy_async_all();  // what other SMs stored is read by tile loads
                const int32_t m0 = g.tm * Cfg::kTileRows + (int)rank * kGemmM, n0 = g.tn * BN + (int)rank * Cfg::kBRows;
                for (int kb = 0; kb < g.kblocks; ++kb) {
                    if (!ptx::mbar_wait_bounded(empty0 + 8 * stage, phase ^ 1u, abort_flag, p.wait_limit_ns)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = smem_base + stage * Cfg::kStageBytes, sb = sa + Cfg::kABytes;
                    if (rank == 0) ptx::mbar_arrive_expect_tx(full0 + 8 * stage, CG * Cfg::kStageBytes);
                    const uint32_t bar = full_base + 8 * stage;
                    if (a_mn) {
#pragma unroll
                        for (int s = 0; s < kGemmM / 64; ++s) tma_load_g<CG>(sa + s * 8192, map_a, m0 + 64 * s, kb * kGemmK, bar);
                    } else {
                        tma_load_g<CG>(sa, map_a, kb * kGemmK, m0, bar);
                    }
                    if (b_mn) {
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
            for (int u = worker; ok && u < n_units; u += workers) {
                const MuonUnit g = muon_unit(p, u);
                if (left_out(g)) continue;
                const bool tall = p.matrices[g.matrix].tall;
                const int kind = g.product % 3;
                const bool a_mn = kind == 0 && tall, b_mn = kind == 0 ? tall : kind == 2 && !tall;
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
                    const uint32_t sa = smem_base + s * Cfg::kStageBytes, sb = sa + Cfg::kABytes;
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
    } else {
        const int e = warp - 2, quarter = warp & 3, strip = e >> 2;
        uint32_t acc = 0, acc_phase = 0;
        const uint32_t release0 = CG == 2 ? map_to_rank(accempty0, 0) : accempty0;
        Tile t;
        t.stage = staging + e * 32 * kStagePitch;
        t.lane = lane;
        t.wide = 2;
        for (int u = worker; u < n_units; u += workers) {
            const MuonUnit g = muon_unit(p, u);
            if (left_out(g)) continue;
            const MuonMatrix &q = p.matrices[g.matrix];
            const int kind = g.product % 3, x = g.product / 3 & 1;
            const bool last = g.product + 1 == p.products;
            const int64_t m = kind == 2 ? q.rows : q.d, n = kind == 2 ? q.cols : q.d;
            t.row0 = (int64_t)g.tm * Cfg::kTileRows + (int)rank * kGemmM + quarter * 32;
            t.rows = (int)min(m - t.row0, (int64_t)32);
            t.col0 = g.tn * BN + strip * Cfg::kColsPerWarp;
            t.cols = (int)min(n - t.col0, (int64_t)1 << 20);
            // what this warp reads was stored by other SMs
            bool ok = true;
            if (lane == 0) ok = muon_wait(p.done + g.matrix, g.need, abort_flag, p.wait_limit_ns);
            if (!__all_sync(0xffffffffu, ok)) break;
            const float keep = 1.0f - p.lr * q.wd, step = p.lr * q.scale * q.down;
            uint32_t hi[16], lo[16];
            auto fetch = [&] {
                if (t.rows <= 0 || t.cols <= 0 || kind == 0) return;
                muon_fetch(hi, kind == 1 ? q.gram : q.x[x], kind == 1 ? q.ldd : q.ldx, t);
                if (kind == 2) muon_fetch(lo, q.lo, q.ldx, t);
            };
            fetch();
            if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(accfull0 + 8 * acc, acc_phase, abort_flag, p.wait_limit_ns))) break;
            ptx::tc_fence_after_sync();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + strip * Cfg::kColsPerWarp;
#pragma unroll 1
            for (int c = 0; c < Cfg::kPieces; ++c) {
                float v[32];
                ptx::tmem_ld_32x32(src + c * kPiece, reinterpret_cast<uint32_t (&)[32]>(v));
                ptx::tmem_ld_wait();
                if (c == Cfg::kPieces - 1) {
                    ptx::tc_fence_before_sync();
                    if (lane == 0) {
                        if (CG == 2)
                            mbar_arrive_cluster(release0 + 8 * acc);
                        else
                            ptx::mbar_arrive(release0 + 8 * acc);
                    }
                }
                if (t.rows > 0 && t.cols > 0) {
                    if (kind == 2) {
                        const float a = kNsA;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 h = unpack2<f16>(hi[i]), l = unpack2<f16>(lo[i]);
                            v[2 * i] = fmaf(a, l.x, fmaf(a, h.x, v[2 * i]));
                            v[2 * i + 1] = fmaf(a, l.y, fmaf(a, h.y, v[2 * i + 1]));
                        }
                        if (last) {
                            if (q.param_type == EGERIA_F32)
                                muon_update<float>(q, v, keep, step, t);
                            else if (q.param_type == EGERIA_BF16)
                                muon_update<bf16>(q, v, keep, step, t);
                            else
                                muon_update<f16>(q, v, keep, step, t);
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                hi[i] = pack2<f16>(v[2 * i], v[2 * i + 1]);
                                const float2 h = unpack2<f16>(hi[i]);
                                lo[i] = pack2<f16>(v[2 * i] - h.x, v[2 * i + 1] - h.y);
                            }
                            muon_store(q.x[x ^ 1], q.ldx, hi, t);
                            muon_store(q.lo, q.ldx, lo, t);
                        }
                    } else if (t.row0 <= t.col0) {
                        if (kind == 0) {
                            const float s = q.down * q.down;
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] *= s;
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 h = unpack2<f16>(hi[i]);
                                v[2 * i] = fmaf(kNsC, v[2 * i], kNsB * h.x);
                                v[2 * i + 1] = fmaf(kNsC, v[2 * i + 1], kNsB * h.y);
                            }
                        }
                        muon_store_symmetric(kind == 0 ? q.gram : q.poly, q.ldd, v, t);
                    }
                }
                t.col0 += kPiece;
                t.cols -= kPiece;
                if (c + 1 < Cfg::kPieces) fetch();
            }
            // the tile's share of this warp is there for the loads of any SM
            fence_proxy_async_all();
            __threadfence();
            __syncwarp();
            if (lane == 0) atomicAdd(p.done + g.matrix, 1);
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
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

}  // namespace ops
}  // namespace egeria
