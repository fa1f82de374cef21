// One AdamW step over many tensors in one launch.
//
//   g = gradient * grad_scale
//   m = beta1 m + (1 - beta1) g            v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr wd) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Memory-bound: every value of p, g, m and v is read once and p, m, v are written once.  The
// tensors are cut into blocks of 256 values; one warp takes a block, 8 consecutive values per
// lane, so that a 16-bit tensor is read in 16-byte and a 32-bit one in 32-byte accesses.  8-bit
// moments have one scale per block, which makes the block's maximum a reduction inside the warp.
//
// 8-bit codes.  A first moment is sign * (c / 127)^2 * scale with c = 0..127, and the ROOT of a second
// moment is (c / 255)^2 * scale with c = 0..255; scale is the largest size in the block.  Squaring the
// code spends the steps where the sizes are: next to the maximum a step is 1.6 % (0.8 %) of the
// value, and the smallest size told from zero is 6e-5 (1.5e-5; 2.4e-10 of the second moment itself).
// The root is kept because the update divides by it.  A second moment that is not zero never gets
// code 0: that would divide a moment by eps alone.
#pragma once
#include "../check.cuh"
#include "common.cuh"

namespace egeria {
namespace ops {

constexpr int kAdamBlock = 256;     // values per scale, and per warp and pass
constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kAdamUnroll = 2;      // blocks a warp has in flight
constexpr int kAdamChunk = kAdamBlock * kAdamWarps * kAdamUnroll;  // values per table entry

struct AdamTensor {
    void *p;
    float *master;       // fp32 copy the step works on, or null
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    float wd;
    int32_t module;      // its entry of the freeze mask, -1 = never frozen
    int32_t index;       // its place in the caller's order: gradient pointer and step count
    int32_t vector;      // p, master, m and v take 16/32-byte accesses
};

struct AdamParams {
    const AdamTensor *tensors;
    const int2 *chunks;          // {tensor, chunk of it}
    const void *const *grads;    // by index
    int32_t *steps;              // by index
    const uint8_t *frozen;       // by module, or null
    const float *grad_scale;     // or null
    int32_t *ticket;
    int32_t *status;
    int32_t n_chunks, n_tensors, n_grads;
    float beta1, beta2, rest1, rest2, eps, lr;
    double ln_beta1, ln_beta2;
};

struct AdamStep {   // what a tensor's values need beside themselves
    float decay, rate, root, eps, beta1, rest1, beta2, rest2, gscale;
};

__device__ __forceinline__ void adam_value(const AdamStep &s, float g, float &p, float &m, float &root_v, float &v) {
    g *= s.gscale;
    m = fmaf(s.beta1, m, s.rest1 * g);
    v = fmaf(s.beta2, v, s.rest2 * g * g);
    root_v = fast_sqrt(v);
    p = fmaf(p, s.decay, -s.rate * m * fast_rcp(fmaf(root_v, s.root, s.eps)));
}

__device__ __forceinline__ float decode_root(float c, float unit) {  // unit = scale / MOST^2
    return c * fabsf(c) * unit;
}

// The codes of a block: inv = MOST^2 / scale (0 for a block of zeros, or one that is not finite), so that
// the code of a size a is sqrt(a * inv) = MOST sqrt(a / scale), rounded to the nearest whole number.
// A scale below 2e-34, where inv would overflow, counts as 2e-34: no such moment moves anything.
// A NaN or an infinity in a block leaves the code 0 and a scale that is not finite, which the next
// step decodes as NaN for the whole block.
template <int MOST>
__device__ __forceinline__ float encode_factor(float top) {
    return top > 0.0f ? fminf((float)(MOST * MOST) * fast_rcp(top), 3.0e38f) : 0.0f;
}
template <int MOST>
__device__ __forceinline__ int encode_root(float a, float inv) {
    return min(__float2int_rn(fast_sqrt(a * inv)), MOST);
}

template <typename P, typename G>
struct AdamBlock {
    Raw8<P> p;
    Raw8<G> g;
    Raw8<float> w;
    Raw8<float> m, v;
    uint2 cm, cv;
    float sm, sv;
};

template <typename P, typename G, bool MASTER, bool SMALL>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const AdamParams a) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float gscale = a.grad_scale ? *a.grad_scale : 1.0f;
    const bool skip_all = !(fabsf(gscale) <= 3.402823466e38f);  // not finite: the whole step is left out

    // consecutive chunks per CTA: its tensor changes rarely
    const int per = (a.n_chunks + gridDim.x - 1) / gridDim.x;
    const int c0 = blockIdx.x * per, c1 = min(c0 + per, a.n_chunks);
    int tensor = -1;
    AdamTensor t;
    AdamStep s;
    const G *grad = nullptr;
    bool live = false, vector = false;
    for (int c = c0; c < c1 && !skip_all; ++c) {
        const int2 chunk = a.chunks[c];
        if (!eg_check(chunk.x >= 0 && chunk.x < a.n_tensors && chunk.y >= 0, a.status, 11, c)) break;
        if (chunk.x != tensor) {
            tensor = chunk.x;
            t = a.tensors[tensor];
            if (!eg_check(t.index >= 0 && t.index < a.n_grads, a.status, 12, tensor)) break;
            live = !(a.frozen && t.module >= 0 && a.frozen[t.module]);
            grad = static_cast<const G *>(a.grads[t.index]);
            vector = t.vector && (reinterpret_cast<uintptr_t>(grad) % (8 * sizeof(G)) == 0);
            // 1 - beta^t = -expm1(t ln beta): the product in 64 bits, so that a beta next to 1 keeps its digits
            const double step = (double)a.steps[t.index] + 1.0;
            const float fix1 = -expm1f((float)(step * a.ln_beta1)), fix2 = -expm1f((float)(step * a.ln_beta2));
            s = AdamStep{1.0f - a.lr * t.wd, a.lr / fix1, rsqrtf(fix2), a.eps, a.beta1, a.rest1, a.beta2, a.rest2, gscale};
        }
        if (!live) continue;
        const int64_t base = (int64_t)chunk.y * kAdamChunk;
        if (vector && base + kAdamChunk <= t.n) {
            AdamBlock<P, G> b[kAdamUnroll];
#pragma unroll
            for (int u = 0; u < kAdamUnroll; ++u) {
                const int64_t at = base + (int64_t)(u * kAdamWarps + warp) * kAdamBlock + lane * 8;
                load8(b[u].g, grad + at);
                if (MASTER)
                    load8(b[u].w, t.master + at);
                else
                    load8(b[u].p, static_cast<const P *>(t.p) + at);
                if (SMALL) {
                    b[u].cm = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(t.m) + at);
                    b[u].cv = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(t.v) + at);
                    b[u].sm = t.m_scale[at / kAdamBlock];
                    b[u].sv = t.v_scale[at / kAdamBlock];
                } else {
                    load8(b[u].m, static_cast<const float *>(t.m) + at);
                    load8(b[u].v, static_cast<const float *>(t.v) + at);
                }
            }
#pragma unroll
            for (int u = 0; u < kAdamUnroll; ++u) {
                const int64_t at = base + (int64_t)(u * kAdamWarps + warp) * kAdamBlock + lane * 8;
                float p[8], g[8], m[8], v[8];
                unpack8(g, b[u].g);
                if (MASTER)
                    unpack8(p, b[u].w);
                else
                    unpack8(p, b[u].p);
                if (SMALL) {
                    const float um = b[u].sm * (1.0f / (127.0f * 127.0f)), uv = b[u].sv * (1.0f / (255.0f * 255.0f));
                    float root[8], top_m = 0.0f, top_v = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t wm = i < 4 ? b[u].cm.x : b[u].cm.y, wv = i < 4 ? b[u].cv.x : b[u].cv.y;
                        const float cm = (float)(int8_t)(wm >> (8 * (i & 3))), cv = (float)((wv >> (8 * (i & 3))) & 0xffu);
                        m[i] = decode_root(cm, um);
                        const float r0 = decode_root(cv, uv);
                        v[i] = r0 * r0;
                        adam_value(s, g[i], p[i], m[i], root[i], v[i]);
                        top_m = max_nan(top_m, fabsf(m[i]));
                        top_v = max_nan(top_v, root[i]);
                    }
                    top_m = warp_max_nan(top_m);
                    top_v = warp_max_nan(top_v);
                    const float im = encode_factor<127>(top_m);
                    const float iv = encode_factor<255>(top_v);
                    uint32_t om[2] = {0u, 0u}, ov[2] = {0u, 0u};
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int cm = encode_root<127>(fabsf(m[i]), im);
                        int cv = encode_root<255>(root[i], iv);
                        if (v[i] > 0.0f) cv = max(cv, 1);
                        om[i >> 2] |= (uint32_t)((m[i] < 0.0f ? -cm : cm) & 0xff) << (8 * (i & 3));
                        ov[i >> 2] |= (uint32_t)cv << (8 * (i & 3));
                    }
                    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.m) + at) = make_uint2(om[0], om[1]);
                    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.v) + at) = make_uint2(ov[0], ov[1]);
                    if (lane == 0) {
                        t.m_scale[at / kAdamBlock] = top_m;
                        t.v_scale[at / kAdamBlock] = top_v;
                    }
                } else {
                    unpack8(m, b[u].m);
                    unpack8(v, b[u].v);
                    float root;
#pragma unroll
                    for (int i = 0; i < 8; ++i) adam_value(s, g[i], p[i], m[i], root, v[i]);
                    store8(static_cast<float *>(t.m) + at, m);
                    store8(static_cast<float *>(t.v) + at, v);
                }
                if (MASTER) store8(t.master + at, p);
                store8(static_cast<P *>(t.p) + at, p);
            }
        } else {
            // the end of a tensor, or one whose pointers take no wide access: value by value, lane-consecutive
            for (int u = 0; u < kAdamUnroll; ++u) {
                const int64_t at0 = base + (int64_t)(u * kAdamWarps + warp) * kAdamBlock;
                if (at0 >= t.n) break;
                float p[8], m[8], v[8], root[8], top_m = 0.0f, top_v = 0.0f;
                const float um = SMALL ? t.m_scale[at0 / kAdamBlock] * (1.0f / (127.0f * 127.0f)) : 0.0f;
                const float uv = SMALL ? t.v_scale[at0 / kAdamBlock] * (1.0f / (255.0f * 255.0f)) : 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int64_t at = at0 + lane + 32 * i;
                    const bool in = at < t.n;
                    const float g = in ? to_f32(grad[at]) : 0.0f;
                    p[i] = !in ? 0.0f : MASTER ? t.master[at] : to_f32(static_cast<const P *>(t.p)[at]);
                    if (SMALL) {
                        m[i] = in ? decode_root((float)static_cast<const int8_t *>(t.m)[at], um) : 0.0f;
                        const float r0 = in ? decode_root((float)static_cast<const uint8_t *>(t.v)[at], uv) : 0.0f;
                        v[i] = r0 * r0;
                    } else {
                        m[i] = in ? static_cast<const float *>(t.m)[at] : 0.0f;
                        v[i] = in ? static_cast<const float *>(t.v)[at] : 0.0f;
                    }
                    adam_value(s, g, p[i], m[i], root[i], v[i]);
                    if (in) {
                        top_m = max_nan(top_m, fabsf(m[i]));
                        top_v = max_nan(top_v, root[i]);
                    }
                }
                float im = 0.0f, iv = 0.0f;
                if (SMALL) {
                    top_m = warp_max_nan(top_m);
                    top_v = warp_max_nan(top_v);
                    im = encode_factor<127>(top_m);
                    iv = encode_factor<255>(top_v);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int64_t at = at0 + lane + 32 * i;
                    if (at >= t.n) continue;
                    if (SMALL) {
                        const int cm = encode_root<127>(fabsf(m[i]), im);
                        int cv = encode_root<255>(root[i], iv);
                        if (v[i] > 0.0f) cv = max(cv, 1);
                        static_cast<int8_t *>(t.m)[at] = (int8_t)(m[i] < 0.0f ? -cm : cm);
                        static_cast<uint8_t *>(t.v)[at] = (uint8_t)cv;
                    } else {
                        static_cast<float *>(t.m)[at] = m[i];
                        static_cast<float *>(t.v)[at] = v[i];
                    }
                    if (MASTER) t.master[at] = p[i];
                    static_cast<P *>(t.p)[at] = from_f32<P>(p[i]);
                }
                if (SMALL && lane == 0) {
                    t.m_scale[at0 / kAdamBlock] = top_m;
                    t.v_scale[at0 / kAdamBlock] = top_v;
                }
            }
        }
    }
    // Every CTA has read the step counts; the last one to get here counts this step.
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = (atomicAdd(a.ticket, 1) == (int)gridDim.x - 1);
    }
    __syncthreads();
    if (!last) return;
    if (threadIdx.x == 0) *a.ticket = 0;
    if (skip_all) return;
    for (int i = threadIdx.x; i < a.n_tensors; i += blockDim.x) {
        const int module = a.tensors[i].module;
        if (!(a.frozen && module >= 0 && a.frozen[module])) a.steps[a.tensors[i].index] += 1;
    }
}

}  // namespace ops
}  // namespace egeria
