// The residual stream between two blocks of a network, in one pass over the rows:
//
//   y = alpha x + gate * N_post(f)        h = N_pre(y)
//
// x is the stream, f what a block made of it, N a layer norm or a root-mean-square norm of the row with
// weights and biases, the gate a vector for all rows, one per group of consecutive rows, or absent.
// y goes on as the stream and h into the next block.  Either norm may be left out.
//
// Memory-bound: forward reads x and f and writes y and h; backward reads dy, dh, y and f and writes dx
// and df.  A row lives in the registers of its team of threads between its load and its stores, so the
// means, the variances (of the differences from the mean, in 32 bits) and both norms cost no second
// read.
//
// Measured at 65536 x 1024 bf16 (floor: the bytes at 6464 GB/s): forward with two layer norms 105 us of 83, with two rms
// norms 91 of 83; backward with two rms norms 152 us of 125, with two layer norms 193 of 125.  Forward is bound by
// instructions (36 a value, two thirds of the issue slots).  Backward a value costs 36 instructions, 48 with means and biases, and
// half of the issue slots are taken: what a row waits for (memory, then its team's sums) is not covered by the 16 warps that the
// registers leave room for.  A row pitch that takes no 16-byte accesses costs 2.4 (forward) and 1.8 times that: 252 and 271 us
// at 1001 columns; widths between the teams' own leave threads idle: forward 283 us at 1280 columns, 239 at 1536, 183
// at 2048, 158 at 5120 (the same bytes), 108 at 4096 and 115 at 8192.
#pragma once
#include <string.h>

#include "../ptx_sm100.cuh"
#include "common.cuh"

namespace egeria {
namespace ops {

struct NormParams {
    const void *x, *f, *gate;              // x: y in the backward pass
    const void *w_post, *b_post, *w_pre, *b_pre;
    void *y, *h;                           // backward: dx, df
    const void *dy, *dh;
    float *stats;                          // [rows][4]: mean and 1/deviation of f, of y
    float *sums;                           // backward: column sums per CTA (see norm_backward_kernel)
    void *dw_post, *db_post, *dw_pre, *db_pre, *dgate;
    int64_t ldx, ldf, ldy, ldh, lddy, lddh;
    int64_t rows, gate_rows;               // gate_rows: rows that share a gate; = rows for one gate
    int64_t cta_rows, extra;               // backward: rows / CTAs and the remainder
    int32_t cols;
    int32_t layer, post, pre;
    int32_t w_float;                       // weights, biases and gate are float, not T
    float alpha, eps, inv_cols;
    int32_t *status;                       // backward, checked build
};

// A team is TEAM threads that hold one row, 8 * VPT values each.  WIDE: the thread's values are
// VPT runs of 8 consecutive ones (16- or 32-byte accesses); else value j of thread t is column
// t + TEAM * j, so that the narrow accesses of a row whose pitch allows no wide ones still coalesce.
template <int TEAM, bool WIDE>
__device__ __forceinline__ int norm_col(int t, int i, int j) {
    return WIDE ? (i * TEAM + t) * 8 + j : (i * 8 + j) * TEAM + t;
}

// Whether value j of run i lies in the row.  FULL: every one does (cols = 8 * TEAM * VPT); WIDE: a run does or does not.
template <int TEAM, bool WIDE, bool FULL>
__device__ __forceinline__ bool norm_in(int t, int i, int j, int cols) {
    return FULL || norm_col<TEAM, WIDE>(t, i, WIDE ? 0 : j) < cols;
}

// Run i of a row; zeros past its end.
template <typename T, int TEAM, bool WIDE, bool FULL>
__device__ __forceinline__ void norm_load(Raw8<T> &d, const T *row, int t, int i, int cols) {
    if (WIDE) {
        if (norm_in<TEAM, WIDE, FULL>(t, i, 0, cols)) {
            load8(d, row + norm_col<TEAM, WIDE>(t, i, 0));
            return;
        }
#pragma unroll
        for (uint32_t &r : d.r) r = 0u;
    } else {
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = norm_col<TEAM, WIDE>(t, i, j);
            v[j] = c < cols ? row[c] : from_f32<T>(0.0f);
        }
        memcpy(&d, v, sizeof(v));
    }
}
template <typename T, int TEAM, bool WIDE, bool FULL>
__device__ __forceinline__ void norm_store(T *row, const F2 (&v)[4], int t, int i, int cols) {
    if (WIDE) {
        if (norm_in<TEAM, WIDE, FULL>(t, i, 0, cols)) store8(row + norm_col<TEAM, WIDE>(t, i, 0), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = norm_col<TEAM, WIDE>(t, i, j);
            const float2 f = split(v[j / 2]);
            if (c < cols) row[c] = from_f32<T>(j % 2 ? f.y : f.x);
        }
    }
}
// A vector of `cols` weights, biases or gates, of type float or T, or `absent` in each place; it stays in L1.
// WIDE: aligned like a row.
template <typename T, int TEAM, bool WIDE, bool FULL>
__device__ __forceinline__ void norm_vector(F2 (&v)[4], const void *p, int64_t first, int is_float, int t, int i, int cols, float absent) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f2(absent);
    } else if (is_float) {
        Raw8<float> d;
        norm_load<float, TEAM, WIDE, FULL>(d, static_cast<const float *>(p) + first, t, i, cols);
        unpack8(v, d);
    } else {
        Raw8<T> d;
        norm_load<T, TEAM, WIDE, FULL>(d, static_cast<const T *>(p) + first, t, i, cols);
        unpack8(v, d);
    }
}

// Sums over the team of N = 1 or 2 values, the same bits in every thread.  `scratch`: 2 x 2 x 32 floats; `turn` alternates
// between its halves, so that one barrier per reduction is enough.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float *scratch, int &turn) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (N == 2) {
        // the half-warps take one value each
        const bool upper = lane & 16;
        float mine = upper ? v[1] : v[0];
        mine += __shfl_xor_sync(0xffffffffu, upper ? v[0] : v[1], 16);
#pragma unroll
        for (int o = 8; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (TEAM == 32) {
            v[0] = __shfl_sync(0xffffffffu, mine, 0);
            v[1] = __shfl_sync(0xffffffffu, mine, 16);
            return;
        }
        v[0] = mine;
    } else {
        v[0] = warp_sum(v[0]);
        if (TEAM == 32) return;
    }
    float *half = scratch + (turn & 1) * 64;
    turn ^= 1;
    if ((lane & (N == 2 ? 15 : 31)) == 0) half[(lane >> 4) * 32 + warp] = v[0];
    __syncthreads();
    if (TEAM <= 256) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = half[n * 32];
#pragma unroll
            for (int w = 1; w < TEAM / 32; ++w) v[n] += half[n * 32 + w];
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = warp_sum(lane < TEAM / 32 ? half[n * 32 + lane] : 0.0f);
    }
}

// Takes the mean off the row that the team holds in v (layer norm) and returns it and 1/deviation.
template <int TEAM, int VPT, bool WIDE, bool FULL>
__device__ __forceinline__ void norm_center(F2 (&v)[VPT][4], const NormParams &p, int t, float &mean, float &inv, float *scratch,
                                            int &turn) {
    mean = 0.0f;
    if (p.layer) {
        F2 s2 = f2(0.0f);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2 = s2 + v[i][j];  // past the row's end there are zeros
        float s[1] = {both(s2)};
        team_sum<TEAM>(s, scratch, turn);
        mean = s[0] * p.inv_cols;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo = norm_in<TEAM, WIDE, FULL>(t, i, 2 * j, p.cols) ? -mean : 0.0f;
                const float hi = norm_in<TEAM, WIDE, FULL>(t, i, 2 * j + 1, p.cols) ? -mean : 0.0f;
                v[i][j] = v[i][j] + f2(lo, hi);
            }
    }
    F2 q2 = f2(0.0f);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) q2 = fma2(v[i][j], v[i][j], q2);
    float q[1] = {both(q2)};
    team_sum<TEAM>(q, scratch, turn);
    inv = rsqrtf(fmaf(q[0], p.inv_cols, p.eps));
}

// A warp per row up to 1024 columns (no barrier at all), 128 threads up to 4096, 256 beyond: wider teams with fewer values
// per thread took 120 us against 107 at 16384 x 4096 and 136 against 115 at 8192 x 8192.
template <typename T, int TEAM, int VPT, bool WIDE, bool FULL>
__global__ void __launch_bounds__(TEAM == 32 ? 128 : TEAM) norm_forward_kernel(const NormParams p) {
    __shared__ float scratch[2 * 32 * 2];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    int turn = 0;
    const int t = TEAM == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const int64_t r = TEAM == 32 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (r >= p.rows) return;
    Raw8<T> rx[VPT], rf[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        norm_load<T, TEAM, WIDE, FULL>(rf[i], static_cast<const T *>(p.f) + r * p.ldf, t, i, p.cols);
        norm_load<T, TEAM, WIDE, FULL>(rx[i], static_cast<const T *>(p.x) + r * p.ldx, t, i, p.cols);
    }
    F2 f[VPT][4];
#pragma unroll
    for (int i = 0; i < VPT; ++i) unpack8(f[i], rf[i]);
    float st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.post) norm_center<TEAM, VPT, WIDE, FULL>(f, p, t, st[0], st[1], scratch, turn);
    const int64_t gate = p.gate ? (r / p.gate_rows) * p.cols : 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        F2 v[4], b[4];
        if (p.post) {
            norm_vector<T, TEAM, WIDE, FULL>(v, p.w_post, 0, p.w_float, t, i, p.cols, 1.0f);
            norm_vector<T, TEAM, WIDE, FULL>(b, p.b_post, 0, p.w_float, t, i, p.cols, 0.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i][j] = fma2(f[i][j] * f2(st[1]), v[j], b[j]);
        }
        if (p.gate) {
            norm_vector<T, TEAM, WIDE, FULL>(v, p.gate, gate, p.w_float, t, i, p.cols, 1.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i][j] = f[i][j] * v[j];
        }
        unpack8(v, rx[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i][j] = fma2(f2(p.alpha), v[j], f[i][j]);  // zeros stay past the row's end: all vectors are 0 there
        norm_store<T, TEAM, WIDE, FULL>(static_cast<T *>(p.y) + r * p.ldy, f[i], t, i, p.cols);
    }
    if (p.pre) {
        norm_center<TEAM, VPT, WIDE, FULL>(f, p, t, st[2], st[3], scratch, turn);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            F2 v[4], b[4];
            norm_vector<T, TEAM, WIDE, FULL>(v, p.w_pre, 0, p.w_float, t, i, p.cols, 1.0f);
            norm_vector<T, TEAM, WIDE, FULL>(b, p.b_pre, 0, p.w_float, t, i, p.cols, 0.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i][j] = fma2(f[i][j] * f2(st[3]), v[j], b[j]);
            norm_store<T, TEAM, WIDE, FULL>(static_cast<T *>(p.h) + r * p.ldh, f[i], t, i, p.cols);
        }
    }
    if (t == 0 && p.stats) *reinterpret_cast<float4 *>(p.stats + 4 * r) = make_float4(st[0], st[1], st[2], st[3]);
}

// Backward, given the gradients dy of y (from the stream) and dh of h:
//
//   t   = dy + N_pre'(dh)                dx = alpha t           dgate = sum_rows t * N_post(f)
//   df  = N_post'(gate * t)              dw = sum_rows (gradient of the norm's output) * (normalised row)
//   N'(d) = inv (d w - mean(d w) - hat mean(d w hat)),  hat = (row - mean) inv;  the rms norm has no first mean
//
// A CTA is one team and takes a run of consecutive rows, so that a thread owns its columns and keeps
// their sums over the run in registers.  At the end it writes them as partial sums; the gate's go out
// at the end of every group of rows: straight into dgate if the whole group was this CTA's, else
// as a partial sum (a CTA has at most two groups that it shares: its first and its last).  A second
// kernel adds the partial sums in a fixed order: results do not depend on timing.
// 512 threads per SM in all (128 registers each): 640 of them at 96 registers spill and took 161 us against 151.
// Partial sums per CTA: 6 x cols: dw_pre, db_pre, dw_post, db_post, first group, last group.
constexpr int kNormSums = 6;

template <typename T>
__device__ __forceinline__ void store_param(void *p, int64_t at, float v, int is_float) {
    if (is_float)
        static_cast<float *>(p)[at] = v;
    else
        static_cast<T *>(p)[at] = from_f32<T>(v);
}

// First row of CTA c, the same split in both kernels: the first `extra` CTAs have one row more than the others.
__device__ __forceinline__ int64_t norm_first_row(const NormParams &p, int c) { return c * p.cta_rows + min((int64_t)c, p.extra); }
// The CTA that has row r.
__device__ __forceinline__ int norm_holder(const NormParams &p, int64_t r) {
    const int64_t longer = p.extra * (p.cta_rows + 1);
    return (int)(r < longer ? r / (p.cta_rows + 1) : p.extra + (r - longer) / p.cta_rows);
}

// Rows on their way: a thread copies its own 8 values of each of the four matrices into shared memory, up to two
// rows ahead, and is the only one to read them, so that no barrier belongs to it.
template <typename T, int TEAM>
__host__ __device__ constexpr int norm_ring_rows() {
    return 3 * 4 * TEAM * (int)sizeof(Raw8<T>) <= 200 * 1024 ? 3 : 1;
}
template <typename T>
__device__ __forceinline__ void copy_ahead(Raw8<T> *dst, const T *src, bool in) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    const int bytes = in ? 16 : 0;  // past the row's end: zeros
#pragma unroll
    for (int k = 0; k < (int)sizeof(Raw8<T>) / 16; ++k)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d + 16 * k), "l"(reinterpret_cast<const char *>(src) + (in ? 16 * k : 0)),
                     "r"(bytes)
                     : "memory");
}

// LAYER: layer norms, which have a mean, and norms with biases (a gradient that is not wanted is not written).
template <typename T, int TEAM, bool WIDE, bool FULL, bool LAYER>
__global__ void __launch_bounds__(TEAM, TEAM >= 512 ? 1 : 512 / TEAM) norm_backward_kernel(const NormParams p) {
    constexpr int kRows = norm_ring_rows<T, TEAM>();
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ float scratch[2 * 32 * 2];
    Raw8<T> *ring = reinterpret_cast<Raw8<T> *>(norm_smem);  // [kRows][4][TEAM]
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    int turn = 0;
    const int t = threadIdx.x;
    const int64_t r0 = norm_first_row(p, blockIdx.x), r1 = norm_first_row(p, blockIdx.x + 1);
    if (!eg_check(r0 >= 0 && r0 < r1 && r1 <= p.rows, p.status, kCheckNormRows, r0)) return;
    float *sums = p.sums + (int64_t)blockIdx.x * kNormSums * p.cols;
    const bool in = norm_in<TEAM, WIDE, FULL>(t, 0, 0, p.cols);
    const int col = norm_col<TEAM, WIDE>(t, 0, 0);

    // this thread's place in each matrix, moved on from row to row
    const int c0 = WIDE && in ? col : 0;
    const T *dy = static_cast<const T *>(p.dy) + r0 * p.lddy + c0, *fr = static_cast<const T *>(p.f) + r0 * p.ldf + c0;
    const T *dh = static_cast<const T *>(p.dh), *yr = static_cast<const T *>(p.x);
    if (p.pre) {
        dh += r0 * p.lddh + c0;
        yr += r0 * p.ldx + c0;
    }
    T *dx = static_cast<T *>(p.y) + r0 * p.ldy, *df = static_cast<T *>(p.h) + r0 * p.ldh;
    int64_t fetched = r0;
    auto fetch = [&](int slot) {
        if (WIDE && fetched < r1) {
            Raw8<T> *to = ring + (slot * 4) * TEAM + t;
            copy_ahead(to, dy, in);
            copy_ahead(to + TEAM, fr, in);
            dy += p.lddy;
            fr += p.ldf;
            if (p.pre) {
                copy_ahead(to + 2 * TEAM, dh, in);
                copy_ahead(to + 3 * TEAM, yr, in);
                dh += p.lddh;
                yr += p.ldx;
            }
            ++fetched;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kRows - 1; ++k) fetch(k);

    F2 w_pre[4], w_post[4], b_post[4], gate[4];
    norm_vector<T, TEAM, WIDE, FULL>(w_pre, p.w_pre, 0, p.w_float, t, 0, p.cols, 1.0f);
    norm_vector<T, TEAM, WIDE, FULL>(w_post, p.w_post, 0, p.w_float, t, 0, p.cols, 1.0f);
    if (LAYER) norm_vector<T, TEAM, WIDE, FULL>(b_post, p.b_post, 0, p.w_float, t, 0, p.cols, 0.0f);
    F2 sw_pre[4], sb_pre[4], sw_post[4], sb_post[4], sg[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sw_pre[j] = sb_pre[j] = sw_post[j] = sb_post[j] = sg[j] = f2(0.0f), gate[j] = f2(1.0f);

    int64_t group = 0, left = 0;  // the gate in force and how many of its rows are to come
    int slot = 0;
    constexpr int kSums = LAYER ? 2 : 1;
    float4 st_next = *reinterpret_cast<const float4 *>(p.stats + 4 * r0);
    for (int64_t r = r0; r < r1; ++r) {
        fetch(slot == 0 ? kRows - 1 : slot - 1);
        Raw8<T> ry, rdh, rdy, rf;
        if (WIDE) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRows - 1) : "memory");
            const Raw8<T> *from = ring + (slot * 4) * TEAM + t;
            rdy = from[0];
            rf = from[TEAM];
            if (p.pre) rdh = from[2 * TEAM], ry = from[3 * TEAM];
            slot = slot + 1 == kRows ? 0 : slot + 1;
        } else {
            norm_load<T, TEAM, WIDE, FULL>(rdy, dy, t, 0, p.cols);
            norm_load<T, TEAM, WIDE, FULL>(rf, fr, t, 0, p.cols);
            dy += p.lddy;
            fr += p.ldf;
            if (p.pre) {
                norm_load<T, TEAM, WIDE, FULL>(rdh, dh, t, 0, p.cols);
                norm_load<T, TEAM, WIDE, FULL>(ry, yr, t, 0, p.cols);
                dh += p.lddh;
                yr += p.ldx;
            }
        }
        const float4 st = st_next;
        if (r + 1 < r1) st_next = *reinterpret_cast<const float4 *>(p.stats + 4 * (r + 1));
        if (p.gate && left == 0) {
            group = r / p.gate_rows;
            left = min((group + 1) * p.gate_rows, p.rows) - r;
            if (!eg_check(group >= 0 && group * p.gate_rows < p.rows && left > 0, p.status, kCheckNormGate, group)) return;
            norm_vector<T, TEAM, WIDE, FULL>(gate, p.gate, group * p.cols, p.w_float, t, 0, p.cols, 1.0f);
        }
        F2 tot[4];
        unpack8(tot, rdy);
        if (p.pre) {
            F2 hat[4], d[4], s0 = f2(0.0f), s1 = f2(0.0f);
            unpack8(hat, ry);
            unpack8(d, rdh);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (LAYER) hat[j] = hat[j] + f2(-st.z);
                hat[j] = hat[j] * f2(st.w);
                sw_pre[j] = fma2(d[j], hat[j], sw_pre[j]);
                if (LAYER) sb_pre[j] = sb_pre[j] + d[j];
                d[j] = d[j] * w_pre[j];
                s0 = fma2(d[j], hat[j], s0);  // d is 0 past the row's end
                if (LAYER) s1 = s1 + d[j];
            }
            float s[kSums];
            s[0] = both(s0);
            if (LAYER) s[kSums - 1] = both(s1);
            team_sum<TEAM>(s, scratch, turn);
            const F2 along = f2(-s[0] * p.inv_cols), lean = f2(p.layer ? -s[kSums - 1] * p.inv_cols : 0.0f), inv = f2(st.w);
#pragma unroll
            for (int j = 0; j < 4; ++j) tot[j] = fma2(inv, fma2(hat[j], along, LAYER ? d[j] + lean : d[j]), tot[j]);
        }
        {
            F2 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = f2(p.alpha) * tot[j];
            norm_store<T, TEAM, WIDE, FULL>(dx, v, t, 0, p.cols);
            dx += p.ldy;
        }
        // the branch f
        F2 hat[4], d[4], s0 = f2(0.0f), s1 = f2(0.0f);
        unpack8(hat, rf);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!FULL) {
                const float2 q = split(tot[j]);
                tot[j] = f2(norm_in<TEAM, WIDE, FULL>(t, 0, 2 * j, p.cols) ? q.x : 0.0f, norm_in<TEAM, WIDE, FULL>(t, 0, 2 * j + 1, p.cols) ? q.y : 0.0f);
            }
            if (p.post) {
                if (LAYER) hat[j] = hat[j] + f2(-st.x);
                hat[j] = hat[j] * f2(st.y);
            }
            sg[j] = fma2(tot[j], LAYER ? fma2(hat[j], w_post[j], b_post[j]) : hat[j] * w_post[j], sg[j]);
            d[j] = tot[j] * gate[j];
            sw_post[j] = fma2(d[j], hat[j], sw_post[j]);
            if (LAYER) sb_post[j] = sb_post[j] + d[j];
            d[j] = d[j] * w_post[j];
            s0 = fma2(d[j], hat[j], s0);
            if (LAYER) s1 = s1 + d[j];
        }
        if (p.post) {
            float s[kSums];
            s[0] = both(s0);
            if (LAYER) s[kSums - 1] = both(s1);
            team_sum<TEAM>(s, scratch, turn);
            const F2 along = f2(-s[0] * p.inv_cols), lean = f2(p.layer ? -s[kSums - 1] * p.inv_cols : 0.0f), inv = f2(st.y);
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = inv * fma2(hat[j], along, LAYER ? d[j] + lean : d[j]);
        }
        norm_store<T, TEAM, WIDE, FULL>(df, d, t, 0, p.cols);
        df += p.ldh;
        // the gate's sums leave at the end of a group and at the end of the run
        if (p.gate && (--left == 0 || r + 1 == r1)) {
            const int64_t g0 = group * p.gate_rows, g1 = min(g0 + p.gate_rows, p.rows);
            const bool whole = g0 >= r0 && g1 <= r1, first = g0 <= r0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = norm_col<TEAM, WIDE>(t, 0, j);
                const float v = j % 2 ? split(sg[j / 2]).y : split(sg[j / 2]).x;
                if (c < p.cols) {
                    if (!whole)
                        sums[(first ? 4 : 5) * (int64_t)p.cols + c] = v;
                    else if (p.dgate)
                        store_param<T>(p.dgate, group * p.cols + c, v, p.w_float);
                }
                if (j % 2) sg[j / 2] = f2(0.0f);
            }
        }
    }
    auto put = [&](int place, const F2(&v)[4]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = norm_col<TEAM, WIDE>(t, 0, j);
            if (c < p.cols) sums[place * (int64_t)p.cols + c] = j % 2 ? split(v[j / 2]).y : split(v[j / 2]).x;
        }
    };
    if (p.dw_pre) put(0, sw_pre);
    if (LAYER && p.db_pre) put(1, sb_pre);
    if (p.dw_post) put(2, sw_post);
    if (LAYER && p.db_post) put(3, sb_post);
}

// The sum over k = first..last of src[k * pitch], 32 columns per block (lane = column), the k dealt to the 32 warps;
// in warp 0.  The order depends on the sizes alone.
constexpr int kSumsThreads = 1024;
template <typename F>
__device__ __forceinline__ float sum_partials(int first, int last, float (*part)[33], F at) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float s = 0.0f;
    int k = first + warp;
    for (; k + 7 * 32 <= last; k += 8 * 32) {  // eight loads in flight
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = at(k + 32 * u);
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
    }
#pragma unroll 4
    for (; k <= last; k += 32) s += at(k);
    part[warp][lane] = s;
    __syncthreads();
    s = 0.0f;
    if (warp == 0) {
#pragma unroll
        for (int w = 0; w < 32; ++w) s += part[w][lane];
    }
    __syncthreads();
    return s;
}

// Adds the partial sums of n CTAs.  blockIdx.y < 4: one of the four sums over all rows.  The other blocks finish the gates
// of groups of rows that several CTAs share, in one of two ways: a warp per CTA that finds a group begun by the
// CTA before it and adds its few parts (kLongGroup CTAs at most share a group), or a block per group.
constexpr int kLongGroup = 32;
template <typename T>
__global__ void __launch_bounds__(kSumsThreads) norm_sums_kernel(const NormParams p, int n, int long_groups) {
    __shared__ float part[32][33];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), cc = min(c, p.cols - 1);
    const bool writes = threadIdx.x < 32 && c < p.cols;
    const int64_t pitch = (int64_t)kNormSums * p.cols;
    if (blockIdx.y < 4) {
        void *const outs[4] = {p.dw_pre, p.db_pre, p.dw_post, p.db_post};
        void *out = outs[blockIdx.y];
        if (!out) return;
        const float *src = p.sums + (int64_t)blockIdx.y * p.cols + cc;
        const float s = sum_partials(0, n - 1, part, [&](int k) { return src[k * pitch]; });
        if (writes) store_param<T>(out, c, s, p.w_float);
        return;
    }
    // a group's part is its first CTA's last group (place 5), unless it begins with that CTA, and every other one's first (4)
    const float *head = p.sums + 4 * (int64_t)p.cols + cc, *tail = head + p.cols;
    if (long_groups) {
        const int64_t group = blockIdx.y - 4, g0 = group * p.gate_rows, g1 = min(g0 + p.gate_rows, p.rows);
        const int first = norm_holder(p, g0), last = norm_holder(p, g1 - 1);
        if (first == last) return;
        if (!eg_check(first >= 0 && first < last && last < n, p.status, kCheckNormGate, group)) return;
        const bool begins = norm_first_row(p, first) == g0;
        const float s = sum_partials(first, last, part, [&](int k) { return (k == first && !begins ? tail : head)[k * pitch]; });
        if (writes) store_param<T>(p.dgate, group * p.cols + c, s, p.w_float);
        return;
    }
    const int k = 1 + ((int)blockIdx.y - 4) * 32 + (threadIdx.x >> 5);
    if (k >= n) return;
    const int64_t mine = norm_first_row(p, k), before = norm_first_row(p, k - 1), group = mine / p.gate_rows, g0 = group * p.gate_rows;
    if (g0 == mine || g0 < before) return;
    const int64_t g1 = min(g0 + p.gate_rows, p.rows);
    if (!eg_check(g0 >= 0 && g0 < g1, p.status, kCheckNormGate, group)) return;
    float s = (g0 == before ? head : tail)[(k - 1) * pitch] + head[k * pitch];
#pragma unroll 4
    for (int j = k + 1; j < n && norm_first_row(p, j) < g1; ++j) s += head[j * pitch];
    if (c < p.cols) store_param<T>(p.dgate, group * p.cols + c, s, p.w_float);
}

}  // namespace ops
}  // namespace egeria
