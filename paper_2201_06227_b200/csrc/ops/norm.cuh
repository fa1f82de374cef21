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
#pragma once
#include <string.h>

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
    int32_t cols;
    int32_t layer, post, pre;
    int32_t w_float;                       // weights, biases and gate are float, not T
    float alpha, eps, inv_cols;
};

// A team is TEAM threads that hold one row, 8 * VPT values each.  WIDE: the thread's values are
// VPT runs of 8 consecutive ones (16- or 32-byte accesses); else value j of thread t is column
// t + TEAM * j, so that the narrow accesses of a row whose pitch allows no wide ones still coalesce.
template <int TEAM, bool WIDE>
__device__ __forceinline__ int norm_col(int t, int i, int j) {
    return WIDE ? (i * TEAM + t) * 8 + j : (i * 8 + j) * TEAM + t;
}

template <typename T, int TEAM, bool WIDE>
__device__ __forceinline__ void norm_load(Raw8<T> &d, const T *row, int t, int i, int cols) {
    if (WIDE) {
        const int c = norm_col<TEAM, WIDE>(t, i, 0);
        if (c < cols) {
            load8(d, row + c);
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
template <typename T, int TEAM, bool WIDE>
__device__ __forceinline__ void norm_store(T *row, const float (&v)[8], int t, int i, int cols) {
    if (WIDE) {
        const int c = norm_col<TEAM, WIDE>(t, i, 0);
        if (c < cols) store8(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = norm_col<TEAM, WIDE>(t, i, j);
            if (c < cols) row[c] = from_f32<T>(v[j]);
        }
    }
}
// A vector of `cols` weights, biases or gates, of type float or T, or `absent` in each place; it stays in L1.
// WIDE: aligned like a row.
template <typename T, int TEAM, bool WIDE>
__device__ __forceinline__ void norm_vector(float (&v)[8], const void *p, int64_t first, int is_float, int t, int i, int cols, float absent) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = absent;
    } else if (is_float) {
        Raw8<float> d;
        norm_load<float, TEAM, WIDE>(d, static_cast<const float *>(p) + first, t, i, cols);
        unpack8(v, d);
    } else {
        Raw8<T> d;
        norm_load<T, TEAM, WIDE>(d, static_cast<const T *>(p) + first, t, i, cols);
        unpack8(v, d);
    }
}

// Sums over the team, the same bits in every thread.  `scratch`: 2 x 32 x N floats; `turn` alternates
// between its halves, so that one barrier per reduction is enough.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float *scratch, int &turn) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = warp_sum(v[n]);
    if (TEAM == 32) return;
    float *half = scratch + (turn & 1) * 32 * 2;
    turn ^= 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) half[n * 32 + warp] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = warp_sum(lane < TEAM / 32 ? half[n * 32 + lane] : 0.0f);
}

// Mean and 1/deviation of the row that the team holds in v.
template <int TEAM, bool WIDE, int VPT>
__device__ __forceinline__ void norm_stats(const float (&v)[VPT][8], const NormParams &p, int t, float &mean, float &inv,
                                           float *scratch, int &turn) {
    mean = 0.0f;
    if (p.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[i][j];  // columns past the row's end hold 0
        team_sum<TEAM>(s, scratch, turn);
        mean = s[0] * p.inv_cols;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = norm_col<TEAM, WIDE>(t, i, j) < p.cols ? v[i][j] - mean : 0.0f;
            q[0] = fmaf(d, d, q[0]);
        }
    team_sum<TEAM>(q, scratch, turn);
    inv = rsqrtf(fmaf(q[0], p.inv_cols, p.eps));
}

template <typename T, int TEAM, int VPT, bool WIDE>
__global__ void __launch_bounds__(TEAM == 32 ? 128 : TEAM) norm_forward_kernel(const NormParams p) {
    __shared__ float scratch[2 * 32 * 2];
    int turn = 0;
    const int t = TEAM == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const int64_t row0 = TEAM == 32 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (row0 >= p.rows) return;
    const int64_t r = row0;
    Raw8<T> rx[VPT], rf[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        norm_load<T, TEAM, WIDE>(rf[i], static_cast<const T *>(p.f) + r * p.ldf, t, i, p.cols);
        norm_load<T, TEAM, WIDE>(rx[i], static_cast<const T *>(p.x) + r * p.ldx, t, i, p.cols);
    }
    float f[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) unpack8(f[i], rf[i]);
    float st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.post) norm_stats<TEAM, WIDE>(f, p, t, st[0], st[1], scratch, turn);
    const int64_t gate = p.gate ? (r / p.gate_rows) * p.cols : 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float v[8], b[8];
        if (p.post) {
            norm_vector<T, TEAM, WIDE>(v, p.w_post, 0, p.w_float, t, i, p.cols, 1.0f);
            norm_vector<T, TEAM, WIDE>(b, p.b_post, 0, p.w_float, t, i, p.cols, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = fmaf((f[i][j] - st[0]) * st[1], v[j], b[j]);
        }
        if (p.gate) {
            norm_vector<T, TEAM, WIDE>(v, p.gate, gate, p.w_float, t, i, p.cols, 1.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] *= v[j];
        }
        unpack8(v, rx[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            f[i][j] = norm_col<TEAM, WIDE>(t, i, j) < p.cols ? fmaf(p.alpha, v[j], f[i][j]) : 0.0f;
        norm_store<T, TEAM, WIDE>(static_cast<T *>(p.y) + r * p.ldy, f[i], t, i, p.cols);
    }
    if (p.pre) {
        norm_stats<TEAM, WIDE>(f, p, t, st[2], st[3], scratch, turn);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float v[8], b[8];
            norm_vector<T, TEAM, WIDE>(v, p.w_pre, 0, p.w_float, t, i, p.cols, 1.0f);
            norm_vector<T, TEAM, WIDE>(b, p.b_pre, 0, p.w_float, t, i, p.cols, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = fmaf((f[i][j] - st[2]) * st[3], v[j], b[j]);
            norm_store<T, TEAM, WIDE>(static_cast<T *>(p.h) + r * p.ldh, f[i], t, i, p.cols);
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
// Partial sums per CTA: 6 x cols: dw_pre, db_pre, dw_post, db_post, first group, last group.
constexpr int kNormSums = 6;

template <typename T>
__device__ __forceinline__ void store_param(void *p, int64_t at, float v, int is_float) {
    if (is_float)
        static_cast<float *>(p)[at] = v;
    else
        static_cast<T *>(p)[at] = from_f32<T>(v);
}

// Rows of CTA c of n: the same split in both kernels.
__host__ __device__ __forceinline__ int64_t norm_first_row(int64_t rows, int n, int c) { return rows * c / n; }

template <typename T, int TEAM, int VPT, bool WIDE>
__global__ void __launch_bounds__(TEAM) norm_backward_kernel(const NormParams p) {
    __shared__ float scratch[2 * 32 * 2];
    int turn = 0;
    const int t = threadIdx.x;
    const int64_t r0 = norm_first_row(p.rows, gridDim.x, blockIdx.x), r1 = norm_first_row(p.rows, gridDim.x, blockIdx.x + 1);
    float sw_pre[VPT][8], sb_pre[VPT][8], sw_post[VPT][8], sb_post[VPT][8], sg[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sw_pre[i][j] = sb_pre[i][j] = sw_post[i][j] = sb_post[i][j] = sg[i][j] = 0.0f;
    float *sums = p.sums + (int64_t)blockIdx.x * kNormSums * p.cols;

    for (int64_t r = r0; r < r1; ++r) {
        Raw8<T> ry[VPT], rdh[VPT], rdy[VPT], rf[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (p.pre) {
                norm_load<T, TEAM, WIDE>(ry[i], static_cast<const T *>(p.x) + r * p.ldx, t, i, p.cols);
                norm_load<T, TEAM, WIDE>(rdh[i], static_cast<const T *>(p.dh) + r * p.lddh, t, i, p.cols);
            }
            norm_load<T, TEAM, WIDE>(rdy[i], static_cast<const T *>(p.dy) + r * p.lddy, t, i, p.cols);
            norm_load<T, TEAM, WIDE>(rf[i], static_cast<const T *>(p.f) + r * p.ldf, t, i, p.cols);
        }
        const float4 st = *reinterpret_cast<const float4 *>(p.stats + 4 * r);
        float tot[VPT][8], v[8];
#pragma unroll
        for (int i = 0; i < VPT; ++i) unpack8(tot[i], rdy[i]);
        if (p.pre) {
            float hat[VPT][8], d[VPT][8], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                unpack8(hat[i], ry[i]);
                unpack8(d[i], rdh[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hat[i][j] = (hat[i][j] - st.z) * st.w;
                    sw_pre[i][j] = fmaf(d[i][j], hat[i][j], sw_pre[i][j]);
                    sb_pre[i][j] += d[i][j];
                }
                norm_vector<T, TEAM, WIDE>(v, p.w_pre, 0, p.w_float, t, i, p.cols, 1.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[i][j] *= v[j];
                    s[0] = fmaf(d[i][j], hat[i][j], s[0]);  // d is 0 past the row's end
                    s[1] += d[i][j];
                }
            }
            team_sum<TEAM>(s, scratch, turn);
            const float along = s[0] * p.inv_cols, lean = p.layer ? s[1] * p.inv_cols : 0.0f;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) tot[i][j] = fmaf(st.w, d[i][j] - lean - hat[i][j] * along, tot[i][j]);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p.alpha * tot[i][j];
            norm_store<T, TEAM, WIDE>(static_cast<T *>(p.y) + r * p.ldy, v, t, i, p.cols);
        }
        // the branch f
        const int64_t group = p.gate ? r / p.gate_rows : 0;
        float hat[VPT][8], d[VPT][8], s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            unpack8(hat[i], rf[i]);
            float w[8], b[8];
            if (p.post) {
                norm_vector<T, TEAM, WIDE>(w, p.w_post, 0, p.w_float, t, i, p.cols, 1.0f);
                norm_vector<T, TEAM, WIDE>(b, p.b_post, 0, p.w_float, t, i, p.cols, 0.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) hat[i][j] = (hat[i][j] - st.x) * st.y;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.0f, b[j] = 0.0f;
            }
            if (p.gate) {
                norm_vector<T, TEAM, WIDE>(v, p.gate, group * p.cols, p.w_float, t, i, p.cols, 1.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sg[i][j] = fmaf(tot[i][j], fmaf(hat[i][j], w[j], b[j]), sg[i][j]);
                    d[i][j] = tot[i][j] * v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = tot[i][j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = norm_col<TEAM, WIDE>(t, i, j) < p.cols;
                d[i][j] = in ? d[i][j] : 0.0f;
                sw_post[i][j] = fmaf(d[i][j], hat[i][j], sw_post[i][j]);
                sb_post[i][j] += d[i][j];
                d[i][j] *= w[j];
                s[0] = fmaf(d[i][j], hat[i][j], s[0]);
                s[1] += d[i][j];
            }
        }
        if (p.post) {
            team_sum<TEAM>(s, scratch, turn);
            const float along = s[0] * p.inv_cols, lean = p.layer ? s[1] * p.inv_cols : 0.0f;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = st.y * (d[i][j] - lean - hat[i][j] * along);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) norm_store<T, TEAM, WIDE>(static_cast<T *>(p.h) + r * p.ldh, d[i], t, i, p.cols);
        // the gate's sums leave at the end of a group and at the end of the run
        if (p.gate && (r + 1 == r1 || (r + 1) % p.gate_rows == 0)) {
            const int64_t g0 = group * p.gate_rows, g1 = min(g0 + p.gate_rows, p.rows);
            const bool whole = g0 >= r0 && g1 <= r1, first = g0 <= r0;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = norm_col<TEAM, WIDE>(t, i, j);
                    if (c < p.cols) {
                        if (whole)
                            store_param<T>(p.dgate, group * p.cols + c, sg[i][j], p.w_float);
                        else
                            sums[(first ? 4 : 5) * (int64_t)p.cols + c] = sg[i][j];
                    }
                    sg[i][j] = 0.0f;
                }
        }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = norm_col<TEAM, WIDE>(t, i, j);
            if (c >= p.cols) continue;
            if (p.dw_pre) sums[c] = sw_pre[i][j];
            if (p.db_pre) sums[(int64_t)p.cols + c] = sb_pre[i][j];
            if (p.dw_post) sums[2 * (int64_t)p.cols + c] = sw_post[i][j];
            if (p.db_post) sums[3 * (int64_t)p.cols + c] = sb_post[i][j];
        }
}

// Adds the partial sums of n CTAs.  blockIdx.y < 4: one of the four sums over all rows; else the group
// of rows that CTA y - 4 finds begun by the CTA before it (if there is one, and that CTA began it).
template <typename T>
__global__ void __launch_bounds__(256) norm_sums_kernel(const NormParams p, int n) {
    __shared__ float part[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    void *const outs[4] = {p.dw_pre, p.db_pre, p.dw_post, p.db_post};
    const int what = blockIdx.y;
    int first = 0, last = n - 1;
    int64_t group = 0, g0 = 0;
    void *out;
    if (what < 4) {
        out = outs[what];
        if (!out) return;
    } else {
        const int k = what - 4;
        if (k == 0 || !p.dgate) return;
        out = p.dgate;
        group = norm_first_row(p.rows, n, k) / p.gate_rows;
        g0 = group * p.gate_rows;
        if (g0 == norm_first_row(p.rows, n, k) || g0 < norm_first_row(p.rows, n, k - 1)) return;
        const int64_t g1 = min(g0 + p.gate_rows, p.rows);
        first = k - 1;
        last = k;
        while (last + 1 < n && norm_first_row(p.rows, n, last + 1) < g1) ++last;
    }
    float s = 0.0f;
    for (int k = first + warp; k <= last; k += 8) {
        const int slot = what < 4 ? what : (g0 <= norm_first_row(p.rows, n, k) ? 4 : 5);
        if (c < p.cols) s += p.sums[((int64_t)k * kNormSums + slot) * p.cols + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < p.cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += part[w][lane];
        store_param<T>(out, group * p.cols + c, s, p.w_float);
    }
}

}  // namespace ops
}  // namespace egeria
