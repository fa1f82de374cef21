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
// Measured on 302 M values (a 24-block, 1024-wide decoder; floor: the bytes at 6464 GB/s), bf16 parameters: moments in 32 bits
// 1049 us of 1029, with fp32 masters 1392 of 1309; in 8 bits 818 to 853 us of 471: there the codes' arithmetic (67
// instructions a value) is as long as the bytes, and two thirds of the issue slots are taken.  Frozen tensors are a prefix as a
// rule, and a CTA owns one run of pieces: with 8 of the 24 blocks frozen 931 us of 873, with 16 613 of 436, with 20 532
// of 218, with 23 494 of 55, the time of the CTAs that have all of their run to do.
//
// 8-bit codes.  A first moment is sign * (c / 127)^2 * scale with c = 0..127, and the ROOT of a second
// moment is (c / 255)^2 * scale with c = 0..255; scale is the largest size in the block.  Squaring the
// code spends the steps where the sizes are: next to the maximum a step is 1.6 % (0.8 %) of the
// value, and the smallest size told from zero is 6e-5 (1.5e-5; 2.4e-10 of the second moment itself).
// The root is kept because the update divides by it.  A second moment that is not zero never gets
// code 0: that would divide a moment by eps alone.
#pragma once
#include "../ptx_sm100.cuh"
#include "common.cuh"

namespace egeria {
namespace ops {

constexpr int kAdamBlock = 256;     // values per scale, and per warp and pass
constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kAdamChunk = kAdamBlock * kAdamWarps;  // values per table entry

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

__device__ __forceinline__ float adam_param(const AdamStep &s, float p, float m, float v) {
    return fmaf(p, s.decay, -s.rate * m * fast_rcp(fmaf(full_sqrt(v), s.root, s.eps)));
}

// A code's byte becomes a float, and a float a code's byte, by the bits of 2^23 + code (1.5 * 2^23 + code): the units that
// convert between the kinds are as slow as those of the roots and would be what the kernel waits for.
__device__ __forceinline__ float code_float(uint32_t word, int i) {  // byte i of word, 0..255
    return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7540 + i)) - 8388608.0f;
}
constexpr float kCodeMagic = 12582912.0f;

// The code of a size is MOST * sqrt(size / top) to the nearest whole number, top the largest in the block, every operation
// rounded in 32 bits.  The approximate units give that number unless they come within 6e-7 MOST of a tie (their errors
// and the formula's own roundings add up to 4.2e-7 MOST); there, once in some thousand values, the correctly rounded
// operations decide.  Codes come out the same wherever the formula is computed operation by operation, so
// that a state can be reproduced bit by bit.
__device__ __noinline__ float exact_code(float size, float top, float most) { return rintf(most * __fsqrt_rn(__fdiv_rn(size, top))); }

__device__ __forceinline__ F2 add_apart(F2 a, F2 b) {
    const float2 x = split(a), y = split(b);
    return f2(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}

// Eight values of a block with moments in codes: the new codes replace the old ones in `wm`, `wv`, the block's new scales
// `sm`, `sv`.  The moments are computed by separately rounded products and sums.
__device__ __forceinline__ void adam_codes(const AdamStep &s, const F2 (&g)[4], F2 (&p)[4], uint32_t (&wm)[2], uint32_t (&wv)[2], float &sm,
                                           float &sv) {
    const F2 um = f2(sm * (1.0f / (127.0f * 127.0f))), uv = f2(sv * (1.0f / (255.0f * 255.0f)));
    const F2 b1 = f2(s.beta1), r1 = f2(s.rest1), b2 = f2(s.beta2), r2 = f2(s.rest2), gs = f2(s.gscale);
    float m[8], v[8], root[8], top_m = 0.0f, top_v = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const F2 gi = g[k] * gs;
        // first moments are stored as two's complement: 128 more is 0..255
        const uint32_t u = wm[k >> 1] ^ 0x80808080u;
        const float lo = code_float(u, 2 * (k & 1)) - 128.0f, hi = code_float(u, 2 * (k & 1) + 1) - 128.0f;
        const F2 cv = f2(code_float(wv[k >> 1], 2 * (k & 1)), code_float(wv[k >> 1], 2 * (k & 1) + 1));
        const F2 old_root = cv * cv * uv;
        // (the sums by themselves: a sum of pairs may be fused with the product before it)
        const F2 mi = add_apart(b1 * (f2(lo * fabsf(lo), hi * fabsf(hi)) * um), r1 * gi);
        const F2 vi = add_apart(b2 * (old_root * old_root), r2 * gi * gi);
        const float2 ms = split(mi), vs = split(vi);
        m[2 * k] = ms.x, m[2 * k + 1] = ms.y, v[2 * k] = vs.x, v[2 * k + 1] = vs.y;
        root[2 * k] = full_sqrt(vs.x), root[2 * k + 1] = full_sqrt(vs.y);
        const float2 d = split(fma2(f2(root[2 * k], root[2 * k + 1]), f2(s.root), f2(s.eps)));
        p[k] = fma2(p[k], f2(s.decay), f2(-s.rate) * mi * f2(fast_rcp(d.x), fast_rcp(d.y)));
        top_m = max_nan(max_nan(top_m, fabsf(ms.x)), fabsf(ms.y));
        top_v = max_nan(max_nan(top_v, vs.x), vs.y);
    }
    sm = warp_max_nan(top_m);
    sv = __fsqrt_rn(warp_max_nan(top_v));
    // an infinity in a block makes its scale NaN, as a NaN does: the next step decodes the whole block to NaN
    if (!(sm <= 3.402823466e38f)) sm = __uint_as_float(0x7fc00000u);
    if (!(sv <= 3.402823466e38f)) sv = __uint_as_float(0x7fc00000u);
    const float im = sm > 0.0f ? 127.0f * 127.0f * fast_rcp(sm) : 0.0f, iv = sv > 0.0f ? 255.0f * 255.0f * fast_rcp(sv) : 0.0f;
    // below these scales the approximate units would take what still has a code for zero, or overflow
    uint32_t ties = (sm > 0.0f && sm < 1e-32f ? 0xffu : 0u) | (sv > 0.0f && sv < 4e-14f ? 0xff00u : 0u);
    float ym[8], yv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float xm = fast_sqrt(fabsf(m[i]) * im), xv = fast_sqrt(root[i] * iv);
        ym[i] = xm + kCodeMagic;
        yv[i] = xv + kCodeMagic;
        if (fabsf(xm - (ym[i] - kCodeMagic)) > 0.5f - 6e-7f * 127.0f) ties |= 1u << i;
        if (fabsf(xv - (yv[i] - kCodeMagic)) > 0.5f - 6e-7f * 255.0f) ties |= 256u << i;
    }
    if (ties) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (ties & (1u << i)) ym[i] = exact_code(fabsf(m[i]), sm, 127.0f) + kCodeMagic;
            if (ties & (256u << i)) yv[i] = exact_code(__fsqrt_rn(v[i]), sv, 255.0f) + kCodeMagic;
        }
    }
    uint32_t bm[8], bv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // the sign goes into the code: 2 * magic - y is magic - code
        bm[i] = __float_as_uint(m[i] < 0.0f ? 2.0f * kCodeMagic - ym[i] : ym[i]);
        bv[i] = __float_as_uint(fmaxf(yv[i], v[i] > 0.0f ? kCodeMagic + 1.0f : kCodeMagic));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        wm[k] = __byte_perm(__byte_perm(bm[4 * k], bm[4 * k + 1], 0x0040), __byte_perm(bm[4 * k + 2], bm[4 * k + 3], 0x0040), 0x5410);
        wv[k] = __byte_perm(__byte_perm(bv[4 * k], bv[4 * k + 1], 0x0040), __byte_perm(bv[4 * k + 2], bv[4 * k + 3], 0x0040), 0x5410);
    }
}

// A block of 256 values in flight: what its lane has loaded of it.
template <typename P, typename G>
struct AdamBlock {
    Raw8<P> p;
    Raw8<G> g;
    Raw8<float> w, m, v;
    uint2 cm, cv;
    float sm, sv;
};
template <typename P, typename G, bool MASTER, bool SMALL>
__device__ __forceinline__ void adam_load(AdamBlock<P, G> &b, const AdamTensor &t, const G *grad, int64_t at) {
    load8(b.g, grad + at);
    if (MASTER)
        load8(b.w, t.master + at);
    else
        load8(b.p, static_cast<const P *>(t.p) + at);
    if (SMALL) {
        b.cm = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(t.m) + at);
        b.cv = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(t.v) + at);
        b.sm = t.m_scale[at / kAdamBlock];
        b.sv = t.v_scale[at / kAdamBlock];
    } else {
        load8(b.m, static_cast<const float *>(t.m) + at);
        load8(b.v, static_cast<const float *>(t.v) + at);
    }
}
template <typename P, typename G, bool MASTER, bool SMALL>
__device__ __forceinline__ void adam_finish(AdamBlock<P, G> &b, const AdamStep &s, const AdamTensor &t, int64_t at, int lane) {
    if (SMALL) {
        F2 p[4], g[4];
        unpack8(g, b.g);
        if (MASTER)
            unpack8(p, b.w);
        else
            unpack8(p, b.p);
        uint32_t wm[2] = {b.cm.x, b.cm.y}, wv[2] = {b.cv.x, b.cv.y};
        adam_codes(s, g, p, wm, wv, b.sm, b.sv);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.m) + at) = make_uint2(wm[0], wm[1]);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.v) + at) = make_uint2(wv[0], wv[1]);
        if (lane == 0) {
            t.m_scale[at / kAdamBlock] = b.sm;
            t.v_scale[at / kAdamBlock] = b.sv;
        }
        if (MASTER) store8(t.master + at, p);
        store8(static_cast<P *>(t.p) + at, p);
        return;
    }
    float p[8], g[8], m[8], v[8];
    unpack8(g, b.g);
    if (MASTER)
        unpack8(p, b.w);
    else
        unpack8(p, b.p);
    unpack8(m, b.m);
    unpack8(v, b.v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = g[i] * s.gscale;
        m[i] = fmaf(s.beta1, m[i], s.rest1 * gi);
        v[i] = fmaf(s.beta2, v[i], s.rest2 * gi * gi);
        p[i] = adam_param(s, p[i], m[i], v[i]);
    }
    store8(static_cast<float *>(t.m) + at, m);
    store8(static_cast<float *>(t.v) + at, v);
    if (MASTER) store8(t.master + at, p);
    store8(static_cast<P *>(t.p) + at, p);
}
// The end of a tensor, or a block of one whose pointers take no wide access: value by value, lane-consecutive.
template <typename P, typename G, bool MASTER, bool SMALL>
__device__ __forceinline__ void adam_narrow(const AdamStep &s, const AdamTensor &t, const G *grad, int64_t at0, int lane) {
    float p[8], g[8], m[8], v[8];
    uint32_t wm[2] = {0u, 0u}, wv[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t at = at0 + lane + 32 * i;
        const bool in = at < t.n;  // zeros stand for what is not there: they stay zeros
        g[i] = in ? to_f32(grad[at]) : 0.0f;
        p[i] = !in ? 0.0f : MASTER ? t.master[at] : to_f32(static_cast<const P *>(t.p)[at]);
        if (SMALL) {
            wm[i >> 2] |= (in ? (uint32_t)static_cast<const uint8_t *>(t.m)[at] : 0u) << (8 * (i & 3));
            wv[i >> 2] |= (in ? (uint32_t)static_cast<const uint8_t *>(t.v)[at] : 0u) << (8 * (i & 3));
        } else {
            m[i] = in ? static_cast<const float *>(t.m)[at] : 0.0f;
            v[i] = in ? static_cast<const float *>(t.v)[at] : 0.0f;
        }
    }
    if (SMALL) {
        float sm = t.m_scale[at0 / kAdamBlock], sv = t.v_scale[at0 / kAdamBlock];
        F2 g2[4], p2[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) g2[k] = f2(g[2 * k], g[2 * k + 1]), p2[k] = f2(p[2 * k], p[2 * k + 1]);
        adam_codes(s, g2, p2, wm, wv, sm, sv);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 q = split(p2[k]);
            p[2 * k] = q.x, p[2 * k + 1] = q.y;
        }
        if (lane == 0) {
            t.m_scale[at0 / kAdamBlock] = sm;
            t.v_scale[at0 / kAdamBlock] = sv;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t at = at0 + lane + 32 * i;
        if (at >= t.n) continue;
        if (SMALL) {
            static_cast<uint8_t *>(t.m)[at] = (uint8_t)(wm[i >> 2] >> (8 * (i & 3)));
            static_cast<uint8_t *>(t.v)[at] = (uint8_t)(wv[i >> 2] >> (8 * (i & 3)));
        } else {
            const float gi = g[i] * s.gscale;
            m[i] = fmaf(s.beta1, m[i], s.rest1 * gi);
            v[i] = fmaf(s.beta2, v[i], s.rest2 * gi * gi);
            p[i] = adam_param(s, p[i], m[i], v[i]);
            static_cast<float *>(t.m)[at] = m[i];
            static_cast<float *>(t.v)[at] = v[i];
        }
        if (MASTER) t.master[at] = p[i];
        static_cast<P *>(t.p)[at] = from_f32<P>(p[i]);
    }
}

// Three CTAs per SM for 8-bit moments (80 registers, a few spilled): 825 us against 924 with two, before the sums of pairs
// were taken apart.
template <typename P, typename G, bool MASTER, bool SMALL>
__global__ void __launch_bounds__(kAdamThreads, SMALL ? 3 : 2) adamw_kernel(const AdamParams a) {
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    // blocks that a warp has in flight: moments in 32 bits are enough bytes with one (302 M bf16 values 1054 us, with two 1108);
    // in 8 bits it takes two (825 us, with one 937, before the sums of pairs were taken apart)
    constexpr int kUnroll = SMALL ? 2 : 1;
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
        if (!eg_check(chunk.x >= 0 && chunk.x < a.n_tensors && chunk.y >= 0, a.status, kCheckAdamPiece, c)) break;
        if (chunk.x != tensor) {
            tensor = chunk.x;
            t = a.tensors[tensor];
            if (!eg_check(t.index >= 0 && t.index < a.n_grads, a.status, kCheckAdamTensor, tensor)) break;
            live = !(a.frozen && t.module >= 0 && a.frozen[t.module]);
            grad = static_cast<const G *>(a.grads[t.index]);
            vector = t.vector && (reinterpret_cast<uintptr_t>(grad) % (8 * sizeof(G)) == 0);
            // 1 - beta^t = -expm1(t ln beta): the product in 64 bits, so that a beta next to 1 keeps its digits
            const double step = (double)a.steps[t.index] + 1.0;
            const float fix1 = -expm1f((float)(step * a.ln_beta1)), fix2 = -expm1f((float)(step * a.ln_beta2));
            s = AdamStep{1.0f - a.lr * t.wd, a.lr / fix1, rsqrtf(fix2), a.eps, a.beta1, a.rest1, a.beta2, a.rest2, gscale};
        }
        if (!live) continue;
        const int64_t at0 = (int64_t)chunk.y * kAdamChunk + warp * kAdamBlock;
        // the next entries go on with the same tensor as a rule: then kUnroll blocks of a warp are in flight together
        const bool more = c + kUnroll <= c1 && a.chunks[c + kUnroll - 1].x == tensor;
        if (vector && more && ((int64_t)chunk.y + kUnroll) * kAdamChunk <= t.n) {
            AdamBlock<P, G> b[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) adam_load<P, G, MASTER, SMALL>(b[u], t, grad, at0 + u * kAdamChunk + lane * 8);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) adam_finish<P, G, MASTER, SMALL>(b[u], s, t, at0 + u * kAdamChunk + lane * 8, lane);
            c += kUnroll - 1;
        } else if (at0 >= t.n) {
            // (nothing of it is this warp's)
        } else if (vector && at0 + kAdamBlock <= t.n) {
            AdamBlock<P, G> b;
            adam_load<P, G, MASTER, SMALL>(b, t, grad, at0 + lane * 8);
            adam_finish<P, G, MASTER, SMALL>(b, s, t, at0 + lane * 8, lane);
        } else {
            adam_narrow<P, G, MASTER, SMALL>(s, t, grad, at0, lane);
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
