// layers_elem.cuh -- element types, activations and the end of a product
// (bias, activation, gate, residual, rounding), shared by the layer kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "layers.h"

namespace vqc {
namespace layers {

// Waits until the kernels before in the stream have ended and their writes are seen: in
// every thread, before any access to memory that another kernel may write.
__device__ __forceinline__ void stream_order() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
// Lets the next kernel of the stream be placed once every CTA has come here: before the
// last stores, not at the start, where its waiting CTAs would take the SMs' room from
// this kernel's later ones.
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half(v); }

// packed float pairs (one instruction for both)
__device__ __forceinline__ unsigned long long pair_bits(float2 a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ float2 pair_of(unsigned long long r) {
    float2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(r));
    return a;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}

__device__ __forceinline__ float exp2f_fast(float x) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// two neighbouring 16-bit elements in a word
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// element i of an array whose type is known at run time (one uniform branch)
__device__ __forceinline__ float load_as(const void* p, int dtype, int64_t i) {
    if (dtype == VQC_F32) return static_cast<const float*>(p)[i];
    if (dtype == VQC_BF16) return to_f(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int dtype, int64_t i, float v) {
    if (dtype == VQC_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == VQC_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16(v);
    else static_cast<__half*>(p)[i] = __float2half(v);
}

// 1 / (1 + exp(-z)), exp by the hardware's power of two: relative error about
// |z| 2^-23, 1 and 0 beyond the range of exp.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.f, 1.f + exp2f_fast(-1.4426950408889634f * z)); }

// The normal distribution function of -a, a = |z|, and exp(-a^2 / 2).
// Phi(-a) = exp(-a^2 / 2) R(a), R(a) = erfcx(a / sqrt 2) / 2 = t P(t), t = 1 / (1 + 0.3 a): P by least
// squares of the relative error, weighted towards its largest (Lawson), 1.7e-7 at most on
// 0 <= a <= 14.5.
// kFull: for float results the exponent's roundings (of a^2, of log2(e) / 2 and of their
// product) are taken along as a factor: both values are good to a relative 2^-20 down to the smallest
// floats.  A result of 16 bits does not show them (8e-6 at a = 12), and they would take 4 of the
// 65 us of 8192 x 2048 x 2048 with residual and z.
template <bool kFull> __device__ __forceinline__ float2 normal_tail(float z) {
    const float a = fminf(fabsf(z), 15.f);      // both are 0 beyond
    const float t = __fdividef(1.f, fmaf(0.3f, a, 1.f));
    float p = fmaf(0.035425145f, t, -0.15616448f);
    p = fmaf(p, t, 0.20456739f);
    p = fmaf(p, t, -0.052043933f);
    p = fmaf(p, t, 0.12769708f);
    p = fmaf(p, t, 0.10017433f);
    p = fmaf(p, t, 0.12071239f);
    p = fmaf(p, t, 0.11963199f);
    const float half_log2e = 0.72134752f, half_log2e_rest = 9.6298149e-9f;
    const float h = a * a, x = -half_log2e * h;
    float e = exp2f_fast(x);
    if (kFull) {
        float r = fmaf(-half_log2e, h, -x);
        r = fmaf(-half_log2e, fmaf(a, a, -h), r);
        r = fmaf(-half_log2e_rest, h, r);
        e = fmaf(e, 0.69314718f * r, e);
    }
    return make_float2(p * t * e, e);
}

// act(z) in float.  A NaN stays one.
template <bool kFull> __device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case VQC_ACT_RELU: return z < 0.f ? 0.f : z;
        case VQC_ACT_GELU: {
            const float q = normal_tail<kFull>(z).x;
            return z * (z < 0.f ? q : 1.f - q);
        }
        case VQC_ACT_SILU: return z * logistic(z);
        case VQC_ACT_TANH: return tanhf(z);
        case VQC_ACT_SIGMOID: return logistic(z);
        default: return z;
    }
}

// act(z) and act'(z)
template <bool kFull> __device__ __forceinline__ float2 act_both(int act, float z) {
    switch (act) {
        case VQC_ACT_RELU: return z < 0.f ? make_float2(0.f, 0.f) : make_float2(z, z == 0.f ? 0.f : 1.f);
        case VQC_ACT_GELU: {
            const float2 t = normal_tail<kFull>(z);
            const float p = z < 0.f ? t.x : 1.f - t.x;
            return make_float2(z * p, fmaf(z, 0.39894228040143268f * t.y, p));
        }
        case VQC_ACT_SILU: {
            const float p = logistic(z);
            return make_float2(z * p, p * fmaf(z, 1.f - p, 1.f));
        }
        case VQC_ACT_TANH: {
            const float a = tanhf(z);
            return make_float2(a, 1.f - a * a);
        }
        case VQC_ACT_SIGMOID: {
            const float p = logistic(z);
            return make_float2(p, p * (1.f - p));
        }
        default: return make_float2(z, 1.f);
    }
}

// The end of a product for W neighbouring elements of a row (1, or 4 where a row holds a
// multiple of 4: outputs are then written at once): v (and u, gated) are the sums.
template <int W>
__device__ __forceinline__ void finish_some(const Finish& f, int which, int64_t row, int64_t col, float (&v)[W], float (&u)[W]) {
    const int64_t at = row * f.n + col;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (f.bias[which]) v[i] += load_as(f.bias[which], f.dtype, col + i);
        if (f.gated && f.bias[1]) u[i] += load_as(f.bias[1], f.dtype, col + i);
    }
    if (f.z[which]) {
        if constexpr (W == 4) {
            *reinterpret_cast<float4*>(f.z[which] + at) = make_float4(v[0], v[1], v[2], v[3]);
            if (f.gated && f.z[1]) *reinterpret_cast<float4*>(f.z[1] + at) = make_float4(u[0], u[1], u[2], u[3]);
        } else {
            f.z[which][at] = v[0];
            if (f.gated && f.z[1]) f.z[1][at] = u[0];
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        v[i] = f.act == kActScale ? v[i] * *f.scale : act_value<true>(f.act, v[i]);
        if (f.gated) v[i] *= u[i];
        if (f.res) v[i] += load_as(f.res, f.out_dtype, row * f.ld_res + col + i);
    }
    if constexpr (W == 4) {
        if (f.out_dtype == VQC_F32) {
            *reinterpret_cast<float4*>(static_cast<float*>(f.y[which]) + at) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            const bool b = f.out_dtype == VQC_BF16;
            const uint2 r = make_uint2(b ? pack2<__nv_bfloat16>(v[0], v[1]) : pack2<__half>(v[0], v[1]),
                                       b ? pack2<__nv_bfloat16>(v[2], v[3]) : pack2<__half>(v[2], v[3]));
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(f.y[which]) + at) = r;
        }
    } else {
        store_as(f.y[which], f.out_dtype, at, v[0]);
    }
}
__device__ __forceinline__ void finish_one(const Finish& f, int which, int64_t row, int64_t col, float v0, float v1) {
    float v[1] = {v0}, u[1] = {v1};
    finish_some<1>(f, which, row, col, v, u);
}

}  // namespace layers
}  // namespace vqc
