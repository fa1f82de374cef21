// Matrix products of the linear layers on the tensor cores, with everything around a product in its epilogue.
//
//   D[m, n] = sum_k A(m, k) B(n, k)         A, B: bf16 or f16 in memory, D accumulated in 32 bits
//
// The three products of a layer differ in which axis of an operand is consecutive in memory:
//   forward  z  = x w^T     A = x  (k consecutive)      B = w  (k consecutive)
//   backward dx = dz w      A = dz (k consecutive)      B = w  (n consecutive)
//   backward dw = dz^T x    A = dz (m consecutive)      B = x  (n consecutive)
// tcgen05 takes either kind from shared memory (one bit per operand), so no operand is ever transposed
// in memory.  Both kinds are staged in 64 x 64 swizzled tiles: a k-consecutive operand as rows of 64 k
// values (128 bytes), the other as rows of 64 m (n) values.
//
// One persistent CTA per SM: warp 0 loads (TMA into a ring of stages of 64 k), warp 1 issues the
// MMAs, the other warps run the epilogue of a tile while the next tile's products go into the other half of
// tensor memory.  One launch takes up to two products (dx and dw of a layer), so that the second fills
// the SMs that the first leaves.  CG = 2: a pair of CTAs shares one tile of 256 rows; each loads its 128 rows of A and
// HALF of B, which is what brings the loads (32 KB per 64 k and CTA instead of 48) near what an SM
// can take from L2 in the time of the MMAs (64 bytes a cycle at their full rate; 60 bytes a nanosecond seen).
//
// Measured (bf16, GPU time in a replayed graph; floor: 2 m n k at 1669 TFLOP/s, a short product's rate; a long run's is 1435
// under the power limit, which these meet too): 65536 x 1024 x 4096 (rows, k, columns) alone 487 us of 329, with bias 533, with
// bias and tanh-gelu 558, with z alone 506, with all of it 576 to 618; k = 4096 and 1024 columns 463 of 329.  dx and dw of
// 16384 x 4096 x 1024 229 to 261 us of 165, with the slope of dx's tanh-gelu 293 to 313.  By the counters no unit is full at
// k = 1024: the tensor pipe is busy for 60 % of the time alone and 51 % with all of the epilogue (67 % alone at k = 4096), L2 for 36
// and 47 %, the issue slots for 16 and 31 %; each part of the epilogue shows in the time although it runs beside the next
// tile's products.  Small products (under some 500 rows) are bound by the 10 us that a launch, its first loads and its one
// epilogue take.
#pragma once
#include <cuda.h>

#include "../ptx_sm100.cuh"
#include "common.cuh"

namespace egeria {
namespace ops {

constexpr int kGemmM = 128;          // rows of D per CTA
constexpr int kGemmK = 64;           // k values per stage: one swizzle row of 128 bytes
constexpr int kEpiWarps = 8;
constexpr int kPiece = 32;           // columns that a warp's epilogue holds at a time (32 rows: one per lane)
constexpr int kStagePitch = 34;      // 16-bit values per row of a warp's 32 x 32 staging tile (odd number of words)

enum { kActNone = 0, kActRelu, kActGelu, kActGeluTanh, kActSilu };

// What is done to a product before it is stored: z = acc + bias (stored if wanted), act(z), then either plus `extra` (a
// residual) or times act_in'(extra).
struct Epilogue {
    const void *bias, *extra;
    void *out, *z;
    int64_t ldx, ldo, ldz;           // pitches of extra, out, z
    int32_t act, act_in;
    int32_t slope;                   // extra is the argument of act_in, not a residual
    int32_t wide;                    // every matrix here takes 32-byte (2), 16-byte (1) or only 2-byte (0) accesses
    int32_t wide_bias;
};
struct GemmProblem {
    CUtensorMap a, b;
    int32_t m, n, kblocks;
    int32_t tiles_m, tiles_n, splits, group_n, units;
    uint32_t a_mn, b_mn;             // the operand's m (n) axis is the consecutive one
    Epilogue epi;
    float *partials;                 // split k: [unit][epilogue warp][piece][8][32 lanes][4]
    int32_t *tickets;                // split k: [tile][epilogue warp], zero between calls
    int64_t partial_floats;          // room for partials (checked build)
    int32_t ticket_room;             // and for tickets
};
// out[c] = the sum of n rows of partial sums.
struct ColumnSums {
    const float *rows;
    void *out;
    int32_t n, cols;
};
struct GemmParams {
    GemmProblem problem[2];
    ColumnSums sums;                 // added up by the epilogue's warps while the first products are computed

    int32_t fill;                    // units of the second product that each worker without a last unit of the first takes before the rest
    uint32_t is_f16;
    uint32_t stall;                  // test hook: the first worker issues no loads (1), or no MMA after its first stage (2)
    int32_t *status;
    uint64_t wait_limit_ns;
};

template <int BN, int CG>
struct GemmCfg {
    static constexpr int kABytes = kGemmM * kGemmK * 2;
    static constexpr int kBRows = BN / CG;                   // rows of B per CTA
    static constexpr int kBBytes = kBRows * kGemmK * 2;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kRing = 192 * 1024;                 // bytes of stages
    static constexpr int kStages = kRing / kStageBytes > 8 ? 8 : kRing / kStageBytes;
    static constexpr int kTmemCols = 2 * BN;
    static constexpr int kThreads = 64 + 32 * kEpiWarps;
    static constexpr int kStaging = kEpiWarps * 32 * kStagePitch * 2;
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kStaging + 256;
    static constexpr int kColsPerWarp = BN / (kEpiWarps / 4);
    static constexpr int kPieces = kColsPerWarp / kPiece;
};

// ---------------------------------------------------------------- PTX of CTA pairs
template <int CG>
__device__ __forceinline__ void tmem_alloc_g(uint32_t dst, uint32_t cols) {
    if (CG == 1)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_free_g(uint32_t addr, uint32_t cols) {
    if (CG == 1) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    }
}
template <int CG>
__device__ __forceinline__ void mma_g(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// One arrival on `bar` (of both CTAs of a pair) once the MMAs issued so far are done.
template <int CG>
__device__ __forceinline__ void mma_commit_g(uint32_t bar) {
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((uint16_t)3)
                     : "memory");
}
// A tile of this CTA; the bytes are counted on `bar`, a barrier of the pair's first CTA.
template <int CG>
__device__ __forceinline__ void tma_load_g(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y)
                     : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(x), "r"(y)
            : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
// The address of `addr` (this CTA's shared memory) in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared-memory descriptor of an operand whose m (n) axis is consecutive: rows of 64 values (128 bytes,
// swizzled), one per k; 8 rows make 1024 bytes (stride offset), the next 64 m values are 64 rows on
// (leading offset).  A step of 16 k is 2048 bytes.
__device__ __forceinline__ uint64_t make_desc_mn_sw128(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((kGemmK * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// ---------------------------------------------------------------- activations
// 1 / (1 + 2^u) from the approximate exponential and reciprocal: relative error below 2e-5 over the range where the
// result is not 0 or 1, far under a 16-bit output's rounding.
__device__ __forceinline__ float logistic2(float u) {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u));
    return fast_rcp(1.0f + e);
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluA = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// Phi(z), the normal distribution, and e = exp(-z^2 / 2), which its density shares.  The tail, Phi(-|z|) = t P(t) e with
// t = 1 / (1 + p |z|) (the form of Hastings' approximations), P the polynomial whose RELATIVE error over |z| <= 13.5 is
// smallest, found by reweighted least squares.  A formula of small absolute error does not do: the value z Phi(z) for
// z < -3 is as small as Phi.  For a value P has degree 5: 4.7e-6, with the roundings of 32 bits and of the exponent 1e-5
// (2^-16.6; a 16-bit result is rounded by 2^-12 of itself at least).  The slope Phi + z e / sqrt(2 pi) is 0 at z = -0.75, where what is
// left of it is the terms' error: there P has degree 7 (1.3e-7), which leaves 1.2e-7, not 1.2e-6.  Values with degree 7 too took
// 595 us against 585 at 65536 x 1024 x 4096 with z; the library's erfcf, which gives more digits than the output holds, 850.
template <bool SLOPE>
__device__ __forceinline__ float normal_cdf(float z, float &e) {
    const float t = fast_rcp(fmaf(SLOPE ? 0.3f : 0.31f, fabsf(z), 1.0f));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-0.5f * kLog2e * (z * z)));
    float q;
    if (SLOPE) {
        q = fmaf(0.0359316915f, t, -0.158275813f);
        q = fmaf(q, t, 0.208206296f);
        q = fmaf(q, t, -0.0553935617f);
        q = fmaf(q, t, 0.129469052f);
        q = fmaf(q, t, 0.0996375382f);
        q = fmaf(q, t, 0.120798349f);
        q = fmaf(q, t, 0.119626388f);
    } else {
        q = fmaf(-0.0739291459f, t, 0.18045035f);
        q = fmaf(q, t, 0.0157447066f);
        q = fmaf(q, t, 0.133429796f);
        q = fmaf(q, t, 0.120441273f);
        q = fmaf(q, t, 0.123860702f);
    }
    const float tail = q * t * e;
    return z < 0.0f ? tail : 1.0f - tail;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == kActRelu) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (ACT == kActGelu) {
        float e;
        return z * normal_cdf<false>(z, e);
    }
    if (ACT == kActGeluTanh) return z * logistic2(z * fmaf(-kLog2e * kGeluA * kGeluB, z * z, -kLog2e * kGeluA));
    if (ACT == kActSilu) return z * logistic2(-kLog2e * z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == kActRelu) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == kActGelu) {
        float e;
        const float phi = normal_cdf<true>(z, e);
        return fmaf(0.39894228040143268f * z, e, phi);
    }
    if (ACT == kActGeluTanh) {
        // p + z p (1 - p) u', u' = A (1 + 3 B z^2).  From |z| = 100 on p is 0 or 1, whatever the square: held there, and with
        // p (1 - p) = 0 as the first factor, no part of the product overflows for a finite z
        const float q = fminf(z * z, 1e4f);
        const float p = logistic2(z * fmaf(-kLog2e * kGeluA * kGeluB, q, -kLog2e * kGeluA));
        return fmaf(p * (1.0f - p) * z, fmaf(3.0f * kGeluA * kGeluB, q, kGeluA), p);
    }
    if (ACT == kActSilu) {
        const float p = logistic2(-kLog2e * z);
        return fmaf(z * p, 1.0f - p, p);
    }
    return 1.0f;
}
template <int N>
__device__ __forceinline__ void act_values(float (&v)[N], int act) {
    switch (act) {
#define EG_ACT(A)                                                        \
    case A:                                                              \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = act_value<A>(v[i]); \
        break;
        EG_ACT(kActRelu)
        EG_ACT(kActGelu)
        EG_ACT(kActGeluTanh)
        EG_ACT(kActSilu)
#undef EG_ACT
    }
}
template <int N>
__device__ __forceinline__ void act_slopes(float (&v)[N], int act) {
    switch (act) {
#define EG_ACT(A)                                                        \
    case A:                                                              \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = act_slope<A>(v[i]); \
        break;
        EG_ACT(kActRelu)
        EG_ACT(kActGelu)
        EG_ACT(kActGeluTanh)
        EG_ACT(kActSilu)
#undef EG_ACT
        default:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 1.0f;
    }
}

// ---------------------------------------------------------------- epilogue of a 32 x 32 piece
// Lane = row; the piece's 32 columns start at col0.  Wide accesses need the whole piece inside the matrix.
__device__ __forceinline__ void ld_v8(uint32_t (&r)[8], const void *p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p));
}
struct Tile {
    int64_t row0;     // first of the warp's 32 rows
    int32_t rows;     // rows of the matrix from row0 on (may exceed 32, or be negative)
    int32_t col0, cols;  // first column of the piece, columns of the matrix from there on
    uint16_t *stage;  // the warp's staging tile
    int lane;
    int wide;
    __device__ __forceinline__ bool fast() const { return wide && cols >= kPiece; }
};
// This lane's row of a piece, as 16 pairs of 16-bit values, by wide loads (zeros for a row that is not there).
__device__ __forceinline__ void piece_fetch(uint32_t (&r)[16], const void *base, int64_t ld, const Tile &t) {
    if (t.lane < t.rows) {
        const uint16_t *p = static_cast<const uint16_t *>(base) + (t.row0 + t.lane) * ld + t.col0;
        if (t.wide == 2) {
            ld_v8(reinterpret_cast<uint32_t (&)[8]>(r[0]), p);
            ld_v8(reinterpret_cast<uint32_t (&)[8]>(r[8]), p + 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 q = *(reinterpret_cast<const uint4 *>(p) + i);
                r[4 * i] = q.x, r[4 * i + 1] = q.y, r[4 * i + 2] = q.z, r[4 * i + 3] = q.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = 0u;
    }
}
// The same for a piece that takes no wide loads: row by row with lane = column, through shared memory.
__device__ __forceinline__ void piece_fetch_narrow(uint32_t (&r)[16], const void *base, int64_t ld, const Tile &t) {
    const int rows = min(t.rows, 32), c = t.lane;
    const uint16_t *p = static_cast<const uint16_t *>(base) + t.row0 * ld + t.col0 + c;
    __syncwarp();
    if (c < t.cols) {
#pragma unroll 8
        for (int k = 0; k < rows; ++k) t.stage[k * kStagePitch + c] = p[k * ld];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = reinterpret_cast<const uint32_t *>(t.stage)[t.lane * (kStagePitch / 2) + i];
}
template <typename T>
__device__ __forceinline__ void piece_store(void *base, int64_t ld, const float (&v)[32], const Tile &t) {
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
    if (t.fast()) {
        if (t.lane < t.rows) {
            T *p = static_cast<T *>(base) + (t.row0 + t.lane) * ld + t.col0;
            if (t.wide == 2) {
                ptx::st_global_v8(reinterpret_cast<float *>(p), r);
                ptx::st_global_v8(reinterpret_cast<float *>(p + 16), r + 8);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(reinterpret_cast<uint4 *>(p) + i) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
            }
        }
        return;
    }
    const int rows = min(t.rows, 32), c = t.lane;
    uint16_t *p = static_cast<uint16_t *>(base) + t.row0 * ld + t.col0 + c;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) reinterpret_cast<uint32_t *>(t.stage)[t.lane * (kStagePitch / 2) + i] = r[i];
    __syncwarp();
    if (c < t.cols) {
#pragma unroll 8
        for (int k = 0; k < rows; ++k) p[k * ld] = t.stage[k * kStagePitch + c];
    }
}
// What the epilogue adds to a piece or takes its slope of.
__device__ __forceinline__ void piece_extra(uint32_t (&r)[16], const Epilogue &p, const Tile &t) {
    if (t.rows <= 0 || t.cols <= 0) return;
    if (t.fast())
        piece_fetch(r, p.extra, p.ldx, t);
    else
        piece_fetch_narrow(r, p.extra, p.ldx, t);
}
// v: the piece's sums; `extra`: what piece_extra fetched.
template <typename T>
__device__ __forceinline__ void piece_finish(const Epilogue &p, float (&v)[32], const uint32_t (&extra)[16], const Tile &t) {
    if (t.rows <= 0 || t.cols <= 0) return;  // the same for the whole warp
    if (p.bias) {
        const T *b = static_cast<const T *>(p.bias) + t.col0;
        if (p.wide_bias && t.cols >= kPiece) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 q = *(reinterpret_cast<const uint4 *>(b) + i);
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = unpack2<T>(w[j]);
                    v[8 * i + 2 * j] += f.x;
                    v[8 * i + 2 * j + 1] += f.y;
                }
            }
        } else {
            const float mine = t.lane < min(t.cols, kPiece) ? to_f32(b[t.lane]) : 0.0f;
#pragma unroll
            for (int i = 0; i < kPiece; ++i) v[i] += __shfl_sync(0xffffffffu, mine, i);
        }
    }
    if (p.z) piece_store<T>(p.z, p.ldz, v, t);
    if (p.act) act_values(v, p.act);
    if (p.extra) {
        if (p.slope) {
            // eight at a time: a slope keeps several registers per value
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float r[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack2<T>(extra[4 * k + i]);
                    r[2 * i] = f.x;
                    r[2 * i + 1] = f.y;
                }
                act_slopes(r, p.act_in);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * k + i] *= r[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = unpack2<T>(extra[i]);
                v[2 * i] += f.x;
                v[2 * i + 1] += f.y;
            }
        }
    }
    piece_store<T>(p.out, p.ldo, v, t);
}

// 32 columns (lane = column) of a column sum by WARPS warps; `part`: WARPS x 33 floats of shared memory, `barrier`: a
// barrier of these warps.
template <typename T, int WARPS, typename B>
__device__ __forceinline__ void add_columns(const ColumnSums &s, int strip, int warp, int lane, float *part, B barrier) {
    const int c = strip * 32 + lane;
    const float *src = s.rows + min(c, s.cols - 1);
    float v = 0.0f;
    int k = warp;
    for (; k + 7 * WARPS < s.n; k += 8 * WARPS) {  // eight loads in flight
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = src[(int64_t)(k + i * WARPS) * s.cols];
#pragma unroll
        for (int i = 0; i < 8; ++i) v += x[i];
    }
#pragma unroll 4
    for (; k < s.n; k += WARPS) v += src[(int64_t)k * s.cols];
    part[warp * 33 + lane] = v;
    barrier();
    if (warp == 0) {
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += part[w * 33 + lane];
        if (c < s.cols) static_cast<T *>(s.out)[c] = from_f32<T>(v);
    }
    barrier();
}

// Unit u: a tile of a product and a range of k blocks.  Tiles go through strips of group_n columns of tiles, n fastest,
// so that the CTAs at work share a few rows of A and a strip of B that stay in L2.
struct GemmUnit {
    int32_t problem, index, tm, tn, tile, split, kb0, kb1;
};
__device__ __forceinline__ GemmUnit gemm_unit(const GemmParams &params, int u) {
    GemmUnit g;
    g.problem = u >= params.problem[0].units;
    g.index = g.problem ? u - params.problem[0].units : u;
    const GemmProblem &p = params.problem[g.problem];
    g.tile = g.index / p.splits;
    g.split = g.index - g.tile * p.splits;
    const int strip = p.group_n * p.tiles_m;
    const int s = g.tile / strip, r = g.tile - s * strip;
    const int w = min(p.group_n, p.tiles_n - s * p.group_n);
    g.tm = r / w;
    g.tn = s * p.group_n + (r - g.tm * w);
    g.kb0 = (int)((int64_t)p.kblocks * g.split / p.splits);
    g.kb1 = (int)((int64_t)p.kblocks * (g.split + 1) / p.splits);
    return g;
}
__device__ __forceinline__ bool gemm_unit_fits(const GemmProblem &q, const GemmUnit &g) {
    return g.tm >= 0 && g.tm < q.tiles_m && g.tn >= 0 && g.tn < q.tiles_n && g.kb0 >= 0 && g.kb0 < g.kb1 && g.kb1 <= q.kblocks;
}
// The step-th unit of a worker (a CTA or a pair), or -1.  The first product's units are dealt round; the workers
// that the last round of it leaves out take `fill` units of the second each, and then that is dealt round.
__device__ __forceinline__ int gemm_next(const GemmParams &p, int worker, int workers, int step) {
    const int first = p.problem[0].units, second = p.problem[1].units;
    const int rounds = first / workers, left = first - rounds * workers;
    const int mine = rounds + (worker < left);
    if (step < mine) return worker + step * workers;
    step -= mine;
    int done = 0;
    if (p.fill) {
        done = (workers - left) * p.fill;
        if (worker >= left) {
            if (step < p.fill) {
                const int u = worker - left + (workers - left) * step;
                return u < second ? first + u : -1;
            }
            step -= p.fill;
        }
    }
    const int64_t u = (int64_t)done + worker + (int64_t)workers * step;
    return u < second ? first + (int)u : -1;
}

template <typename T, int BN, int CG>
__global__ void __launch_bounds__(GemmCfg<BN, CG>::kThreads, 1) gemm_kernel(const __grid_constant__ GemmParams p) {
    using Cfg = GemmCfg<BN, CG>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    uint16_t *staging = reinterpret_cast<uint16_t *>(smem + Cfg::kStages * Cfg::kStageBytes);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Cfg::kStages * Cfg::kStageBytes + Cfg::kStaging);
    const uint32_t full0 = ptx::smem_u32(bars), empty0 = full0 + 8 * Cfg::kStages;
    const uint32_t accfull0 = empty0 + 8 * Cfg::kStages, accempty0 = accfull0 + 16, drain = accempty0 + 16;
    volatile uint32_t *tmem_holder = reinterpret_cast<volatile uint32_t *>(bars + 2 * Cfg::kStages + 5);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    volatile uint32_t *issued = tmem_holder + 2;  // stages that warp 0 has asked for, once it is through
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
        ptx::prefetch_tensormap(&p.problem[0].a);
        ptx::prefetch_tensormap(&p.problem[0].b);
    }
    if (warp == 1) tmem_alloc_g<CG>(ptx::smem_u32(const_cast<uint32_t *>(tmem_holder)), Cfg::kTmemCols);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) cluster_sync();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_holder;
    // Up to here nothing depends on the kernel before this one, which may still be running; from here on everything does.
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, asked = 0;
            bool ok = !(p.stall == 1 && worker == 0);
            // the pair's bytes are counted on its first CTA's barriers
            const uint32_t full_base = CG == 2 ? map_to_rank(full0, 0) : full0;
            for (int step = 0; ok; ++step) {
                const int u = gemm_next(p, worker, workers, step);
                if (u < 0) break;
                const GemmUnit g = gemm_unit(p, u);
                const GemmProblem &q = p.problem[g.problem];
                if (!eg_check(gemm_unit_fits(q, g), p.status, kCheckGemmUnit, u)) break;
                const CUtensorMap *map_a = &q.a, *map_b = &q.b;
                const bool a_mn = q.a_mn, b_mn = q.b_mn;
                const int32_t m0 = (g.tm * CG + (int)rank) * kGemmM, n0 = g.tn * BN + (int)rank * Cfg::kBRows;
                for (int kb = g.kb0; kb < g.kb1; ++kb) {
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
                        for (int s = 0; s < Cfg::kBRows / 64; ++s)
                            tma_load_g<CG>(sb + s * 8192, map_b, n0 + 64 * s, kb * kGemmK, bar);
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
            const uint32_t idesc0 = (1u << 4) | (p.is_f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(BN >> 3) << 17) |
                                    ((uint32_t)((kGemmM * CG) >> 4) << 24);
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
            bool ok = true;
            const bool stop = p.stall == 2 && worker == 0;
            for (int step = 0; ok; ++step) {
                const int u = gemm_next(p, worker, workers, step);
                if (u < 0) break;
                const GemmUnit g = gemm_unit(p, u);
                const GemmProblem &q = p.problem[g.problem];
                if (!ptx::mbar_wait_bounded(accempty0 + 8 * acc, acc_phase ^ 1u, abort_flag, p.wait_limit_ns)) {
                    ok = false;
                    break;
                }
                ptx::tc_fence_after_sync();
                const uint32_t d = tmem + acc * BN;
                const uint32_t idesc = idesc0 | (q.a_mn << 15) | (q.b_mn << 16);
                const uint32_t step_a = q.a_mn ? 2048u >> 4 : 32u >> 4, step_b = q.b_mn ? 2048u >> 4 : 32u >> 4;
                const uint64_t base_a = q.a_mn ? make_desc_mn_sw128(0) : ptx::make_desc_k_sw128(0);
                const uint64_t base_b = q.b_mn ? make_desc_mn_sw128(0) : ptx::make_desc_k_sw128(0);
                const int kb1 = stop ? g.kb0 + 1 : g.kb1;
                for (int kb = g.kb0; kb < kb1; ++kb) {
                    if (!ptx::mbar_wait_bounded(full0 + 8 * stage, phase, abort_flag, p.wait_limit_ns)) {
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t sa = smem_base + stage * Cfg::kStageBytes, sb = sa + Cfg::kABytes;
                    const uint64_t da = base_a | (sa >> 4), db = base_b | (sb >> 4);  // (a CTA's shared window ends below 2^18)
#pragma unroll
                    for (int k = 0; k < kGemmK / 16; ++k)
                        mma_g<CG>(d, da + k * step_a, db + k * step_b, idesc, (kb > g.kb0 || k > 0) ? 1u : 0u);
                    mma_commit_g<CG>(empty0 + 8 * stage);
                    if (++stage == Cfg::kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (stop) ok = false;
                if (!ok) break;
                mma_commit_g<CG>(accfull0 + 8 * acc);
                acc ^= 1u;
                if (acc == 0) acc_phase ^= 1u;
            }
            if (!ok) {
                // gave up: no MMA of ours may still read shared memory when the CTA leaves
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
        if (p.sums.out) {
            for (int c = blockIdx.x; c * 32 < p.sums.cols; c += gridDim.x)
                add_columns<T, kEpiWarps>(p.sums, c, e, lane, reinterpret_cast<float *>(staging),
                                               [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory"); });
        }
        Tile t;
        t.stage = staging + e * 32 * kStagePitch;
        t.lane = lane;
        for (int step = 0;; ++step) {
            const int u = gemm_next(p, worker, workers, step);
            if (u < 0) break;
            const GemmUnit g = gemm_unit(p, u);
            if (!eg_check(gemm_unit_fits(p.problem[g.problem], g), p.status, kCheckGemmUnit, u)) break;
            // (each product with its own copy of this code: what it takes from the parameters is then at fixed places)
            auto tile = [&](const GemmProblem &q) {
                t.wide = q.epi.wide;
                t.row0 = (int64_t)(g.tm * CG + (int)rank) * kGemmM + quarter * 32;
                t.rows = (int)min((int64_t)q.m - t.row0, (int64_t)1 << 20);
                const int col0 = g.tn * BN + strip * Cfg::kColsPerWarp;
                t.col0 = col0;
                t.cols = q.n - col0;
                // what the first piece reads is on its way while the products are computed
                uint32_t extra[16];
                const bool ahead = q.epi.extra && q.splits == 1;
                if (ahead) piece_extra(extra, q.epi, t);
                if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(accfull0 + 8 * acc, acc_phase, abort_flag, p.wait_limit_ns))) return false;
                ptx::tc_fence_after_sync();
                const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + strip * Cfg::kColsPerWarp;
                float *part = nullptr;
                if (q.splits > 1)
                    part = q.partials + (((int64_t)g.index * CG + rank) * kEpiWarps + e) * (Cfg::kPieces * 1024);
                if (q.splits > 1 && !eg_check(part + Cfg::kPieces * 1024 <= q.partials + q.partial_floats &&
                                                  (g.tile * CG + (int)rank) * kEpiWarps + e < q.ticket_room,
                                              p.status, kCheckGemmSplit, g.index))
                    return false;
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
                    if (q.splits > 1) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            *reinterpret_cast<float4 *>(part + ((c * 8 + j) * 32 + lane) * 4) =
                                make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    } else {
                        piece_finish<T>(q.epi, v, extra, t);
                        t.col0 += kPiece;
                        t.cols -= kPiece;
                        if (c + 1 < Cfg::kPieces && ahead) piece_extra(extra, q.epi, t);
                    }
                }
                if (q.splits > 1) {
                    // the last of the tile's splits adds them all, in order, for the part of the tile that is this warp's
                    int done = 0;
                    int32_t *ticket = q.tickets + ((int64_t)(g.tile * CG + (int)rank)) * kEpiWarps + e;
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) done = atomicAdd(ticket, 1);
                    done = __shfl_sync(0xffffffffu, done, 0);
                    if (done == q.splits - 1) {
                        __threadfence();
                        const float *first = q.partials + (((int64_t)g.tile * q.splits * CG + rank) * kEpiWarps + e) * (Cfg::kPieces * 1024);
                        const int64_t pitch = (int64_t)CG * kEpiWarps * Cfg::kPieces * 1024;
#pragma unroll 1
                        for (int c = 0; c < Cfg::kPieces; ++c) {
                            if (q.epi.extra) piece_extra(extra, q.epi, t);
                            float v[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                            for (int s = 0; s < q.splits; ++s) {
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    const float4 f = __ldcg(reinterpret_cast<const float4 *>(first + s * pitch + ((c * 8 + j) * 32 + lane) * 4));
                                    v[4 * j] += f.x, v[4 * j + 1] += f.y, v[4 * j + 2] += f.z, v[4 * j + 3] += f.w;
                                }
                            }
                            piece_finish<T>(q.epi, v, extra, t);
                            t.col0 += kPiece;
                            t.cols -= kPiece;
                        }
                        if (lane == 0) *ticket = 0;
                    }
                }
                return true;
            };
            if (!(g.problem == 0 ? tile(p.problem[0]) : tile(p.problem[1]))) break;
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) {
        // one of the roles gave up: no copy that warp 0 asked for, whichever role that was, may land after this CTA has left
        const uint64_t t0 = ptx::globaltimer_ns();
        if (rank == 0) {
            const uint32_t asked = *issued;
            for (uint32_t k = 1; k <= min(asked, (uint32_t)Cfg::kStages); ++k) {
                const uint32_t idx = asked - k, s = idx % Cfg::kStages, ph = (idx / Cfg::kStages) & 1u;
                while (!ptx::mbar_try_wait(full0 + 8 * s, ph))
                    if (ptx::globaltimer_ns() - t0 > p.wait_limit_ns) break;
            }
        } else {
            // (this CTA's are counted on the other's barriers: a millisecond is a thousand times what one takes)
            while (ptx::globaltimer_ns() - t0 < 1000000ull) {
            }
        }
        atomicMax(p.status, 6);
    }
    if (CG == 2) cluster_sync();
    ptx::tc_fence_after_sync();
    if (warp == 1) tmem_free_g<CG>(tmem, Cfg::kTmemCols);
}

// ---------------------------------------------------------------- a few rows
// y for 1 to 4 rows without the tensor cores: the cost is reading w once, so w is streamed by
// every warp of the GPU in 16-byte pieces, one output column per warp and turn; x stays in shared memory.
// 1024 x 4096: 3.7 us for one row, 6.5 for two, 9.0 for four; the tensor cores take 10 for any number from 5 to 128.
template <typename T, int ROWS, bool WIDE>
__global__ void __launch_bounds__(256) linear_few_kernel(const Epilogue p, int32_t m, int32_t n_cols, const T *x, int64_t ldx, const T *w, int64_t ldw,
                                                         int32_t k) {
    extern __shared__ uint8_t smem_few[];
    T *xs = reinterpret_cast<T *>(smem_few);  // [ROWS][k rounded up to 256], zero behind k
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int kp = (k + 255) & ~255;
    const int rows = min(ROWS, m);
    for (int i = threadIdx.x; i < ROWS * kp; i += blockDim.x) {
        const int r = i / kp, c = i - r * kp;
        xs[i] = (r < rows && c < k) ? x[r * ldx + c] : from_f32<T>(0.0f);
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * 8;
    // (unsigned: past the last of 2^31 - 1024 columns a warp's next turn needs the 32nd bit)
    for (uint32_t n = blockIdx.x * 8 + (threadIdx.x >> 5); n < (uint32_t)n_cols; n += warps) {
        const T *wr = w + (int64_t)n * ldw;
        float acc[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) acc[r] = 0.0f;
        if (WIDE) {
#pragma unroll 4
            for (int c = lane * 8; c < k; c += 256) {  // k is a multiple of 8 here
                Raw8<T> q;
                load8(q, wr + c);
                float wv[8], xv[8];
                unpack8(wv, q);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    Raw8<T> s = *reinterpret_cast<const Raw8<T> *>(xs + r * kp + c);
                    unpack8(xv, s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r] = fmaf(wv[i], xv[i], acc[r]);
                }
            }
        } else {
#pragma unroll 8
            for (int c = lane; c < k; c += 32) {
                const float wv = to_f32(wr[c]);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) acc[r] = fmaf(wv, to_f32(xs[r * kp + c]), acc[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) acc[r] = warp_sum(acc[r]);
        float v[1] = {0.0f};
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (lane == r) v[0] = acc[r];
        if (lane < rows) {
            if (p.bias) v[0] += to_f32(static_cast<const T *>(p.bias)[n]);
            if (p.z) static_cast<T *>(p.z)[lane * p.ldz + n] = from_f32<T>(v[0]);
            act_values(v, p.act);
            if (p.extra) v[0] += to_f32(static_cast<const T *>(p.extra)[lane * p.ldx + n]);
            static_cast<T *>(p.out)[lane * p.ldo + n] = from_f32<T>(v[0]);
        }
    }
}

// ---------------------------------------------------------------- before the products
// One launch does what the products of a call need beforehand: copies of operands whose pitch or address no tile
// load takes, and dz = dy * act'(z) with its column sums.
struct PackJob {
    uint16_t *dst;                   // [rows][pitch]
    const uint16_t *src;             // [rows][ld]
    int64_t pitch, ld, rows, cols;
    int32_t strips, blocks;          // strips of 256 columns; blocks = strips * runs of rows, 0 = nothing to do
};
struct SlopeJob {
    void *dz;                        // or null: only the sums
    const void *dy, *z;              // z null: dz = dy
    float *sums;                     // partial sums [runs][cols], or null
    void *db;                        // the column sums themselves where there is one run
    int64_t lddz, lddy, ldz, rows;
    int64_t sums_room;               // values that sums has room for (checked build)
    int32_t act, cols, strips, runs; // blocks = strips * runs
};
struct PrepareParams {
    SlopeJob slope;
    PackJob pack[2];
    int32_t *status;
};

// A warp owns 256 columns, 8 per lane; the warps of a block take the rows of its run in turn and add up at the end.
// dz is rounded to the operands' type, which is the only one that the products take; the column sums are of dz before that.
// Against one rounding of the results this is a second one where there is an activation: dx and dw of f16 777 x 515 <- 1001
// behind a gelu are off by 2.9e-4 (root mean square, of the values') instead of 2.1e-4; without one, or with relu, whose
// slopes are exact, nothing is added.  Two operands, the rounding and what it leaves, would double the products' time.
// WIDE: a lane's 8 columns are consecutive; else they are 32 apart.
constexpr int kPrepareWarps = 8;
template <typename T, bool WIDE>
__device__ __forceinline__ void slope_block(const SlopeJob &j, int block, float (*part)[256 + 8], int32_t *status) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int run = block / j.strips, c0 = (block - run * j.strips) * 256, cols = j.cols;
    const int64_t r0 = j.rows * run / j.runs, r1 = j.rows * (run + 1) / j.runs;
    const T *dy = static_cast<const T *>(j.dy), *z = static_cast<const T *>(j.z);
    T *dz = static_cast<T *>(j.dz);
    if (!eg_check(run < j.runs && r0 >= 0 && r1 <= j.rows && (!j.sums || j.runs == 1 || (int64_t)(run + 1) * cols <= j.sums_room), status, kCheckSlopeRun, block))
        return;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (WIDE) {
        const int c = c0 + lane * 8;
        if (c < cols) {
            auto row = [&](Raw8<T> &q, Raw8<T> &y, int64_t r) {
                float g[8], a[8];
                unpack8(g, q);
                if (z) {
                    unpack8(a, y);
                    act_slopes(a, j.act);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] *= a[i];
                    if (dz) store8(dz + r * j.lddz + c, g);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += g[i];
            };
            int64_t r = r0 + warp;
            for (; r + 3 * kPrepareWarps < r1; r += 4 * kPrepareWarps) {  // four rows in flight
                Raw8<T> q[4], y[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    load8(q[u], dy + (r + u * kPrepareWarps) * j.lddy + c);
                    if (z) load8(y[u], z + (r + u * kPrepareWarps) * j.ldz + c);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) row(q[u], y[u], r + u * kPrepareWarps);
            }
            for (; r < r1; r += kPrepareWarps) {
                Raw8<T> q, y;
                load8(q, dy + r * j.lddy + c);
                if (z) load8(y, z + r * j.ldz + c);
                row(q, y, r);
            }
        }
    } else {
        for (int64_t r = r0 + warp; r < r1; r += kPrepareWarps) {
            float g[8], a[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0 + lane + 32 * i;
                g[i] = c < cols ? to_f32(dy[r * j.lddy + c]) : 0.0f;
                a[i] = z && c < cols ? to_f32(z[r * j.ldz + c]) : 0.0f;
            }
            if (z) {
                act_slopes(a, j.act);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= a[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0 + lane + 32 * i;
                if (dz && c < cols) dz[r * j.lddz + c] = from_f32<T>(g[i]);
                s[i] += g[i];
            }
        }
    }
    if (!j.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][WIDE ? lane * 8 + i : lane + 32 * i] = s[i];
    __syncthreads();
    const int c = c0 + threadIdx.x;
    if (c < cols) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kPrepareWarps; ++w) v += part[w][threadIdx.x];
        if (j.runs == 1)
            static_cast<T *>(j.db)[c] = from_f32<T>(v);
        else
            j.sums[(int64_t)run * cols + c] = v;
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(32 * kPrepareWarps) prepare_kernel(const PrepareParams p) {
    __shared__ float part[kPrepareWarps][256 + 8];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    int block = blockIdx.x;
    const int slopes = p.slope.strips * p.slope.runs;
    if (block < slopes) {
        slope_block<T, WIDE>(p.slope, block, part, p.status);
        return;
    }
    block -= slopes;
    const PackJob &j = block < p.pack[0].blocks ? p.pack[0] : p.pack[1];
    if (block >= p.pack[0].blocks) block -= p.pack[0].blocks;
    const int run = block / j.strips, runs = j.blocks / j.strips;
    const int64_t c = (int64_t)(block - run * j.strips) * 256 + threadIdx.x;
    if (c >= j.cols) return;
    const int64_t r1 = j.rows * (run + 1) / runs;
#pragma unroll 8
    for (int64_t r = j.rows * run / runs; r < r1; ++r) j.dst[r * j.pitch + c] = j.src[r * j.ld + c];
}

// Column sums on their own, where no product follows that would add them up.
template <typename T>
__global__ void __launch_bounds__(512) add_columns_kernel(const ColumnSums s) {
    __shared__ float part[16 * 33];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    add_columns<T, 16>(s, blockIdx.x, threadIdx.x >> 5, threadIdx.x & 31, part, [] { __syncthreads(); });
}

}  // namespace ops
}  // namespace egeria
