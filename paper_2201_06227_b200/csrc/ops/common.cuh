// What the training operators share: element types, 32-byte accesses, reductions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../check.cuh"

namespace egeria {
namespace ops {

// What the operators' kernels check of themselves in the checked build (the evaluation's codes end at 10).
enum OpsCheckCode : int32_t {
    kCheckAdamPiece = 11,   // AdamW: a table entry's tensor or piece
    kCheckAdamTensor = 12,  // AdamW: a tensor's place in the caller's order
    kCheckGemmUnit = 13,    // products: a unit's tile or range of k blocks
    kCheckGemmSplit = 14,   // products: a split tile's ticket or place among the partial tiles
    kCheckSlopeRun = 15,    // linear backward: a block's rows, or the place of its partial sums
    kCheckNormRows = 16,    // norm backward: a CTA's rows
    kCheckNormGate = 17,    // norm backward: a group's gate, or the CTAs that share it
};

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(f16 v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ f16 from_f32<f16>(float v) { return __float2half_rn(v); }

// Two 32-bit values as one register of a 16-bit type (a in the low half).
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<bf16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<f16>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack2<bf16>(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<f16>(uint32_t v) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

// Eight consecutive values as loaded: 16 bytes of a 16-bit type, 32 bytes of float.  The load and
// the conversion are apart so that several loads can be in flight before the first is used.
template <typename T>
struct alignas(16) Raw8 {
    uint32_t r[sizeof(T) * 2];
};
__device__ __forceinline__ void load8(Raw8<float> &d, const float *p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(d.r[0]), "=r"(d.r[1]), "=r"(d.r[2]), "=r"(d.r[3]), "=r"(d.r[4]), "=r"(d.r[5]), "=r"(d.r[6]),
                   "=r"(d.r[7])
                 : "l"(p));
}
template <typename T>
__device__ __forceinline__ void load8(Raw8<T> &d, const T *p) {
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(d.r[0]), "=r"(d.r[1]), "=r"(d.r[2]), "=r"(d.r[3])
                 : "l"(p));
}
__device__ __forceinline__ void unpack8(float (&v)[8], const Raw8<float> &d) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(d.r[i]);
}
template <typename T>
__device__ __forceinline__ void unpack8(float (&v)[8], const Raw8<T> &d) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(d.r[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(__float_as_uint(v[0])),
                 "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
                 "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])),
                 "r"(__float_as_uint(v[7]))
                 : "memory");
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(pack2<T>(v[0], v[1])),
                 "r"(pack2<T>(v[2], v[3])), "r"(pack2<T>(v[4], v[5])), "r"(pack2<T>(v[6], v[7]))
                 : "memory");
}

// Pairs of floats: one instruction for two products, sums or fused products.  The compiler may fuse a product and a sum of
// pairs in spite of their .rn; where each has to be rounded by itself the sum is taken apart.
struct F2 {
    uint64_t v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 split(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float both(F2 a) {
    const float2 f = split(a);
    return f.x + f.y;
}
template <typename T>
__device__ __forceinline__ void unpack8(F2 (&v)[4], const Raw8<T> &d) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(d.r[i]);
        v[i] = f2(f.x, f.y);
    }
}
__device__ __forceinline__ void unpack8(F2 (&v)[4], const Raw8<float> &d) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(__uint_as_float(d.r[2 * i]), __uint_as_float(d.r[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const F2 (&v)[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 q = split(v[i]);
        f[2 * i] = q.x;
        f[2 * i + 1] = q.y;
    }
    store8(p, f);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Largest of non-negative values; a NaN anywhere gives NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The approximate unit's square root and reciprocal (about one unit in the last place); inputs
// below 2^-126 count as zero.
__device__ __forceinline__ float fast_sqrt(float v) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// The same with inputs below 2^-126 as they are.
__device__ __forceinline__ float full_sqrt(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float fast_rcp(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

}  // namespace ops
}  // namespace egeria
