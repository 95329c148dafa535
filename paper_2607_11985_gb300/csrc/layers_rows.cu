// layers_rows.cu -- products with few rows (single tokens, small batches): the
// weights are all there is to read; they stream through registers once (5 to 16 rows of float:
// once for every four rows).
//
// Up to 4 rows of any type and layout (up to 16 of float, four at a time), FP32
// units: a group of KW warps takes four rows of weights (two of each in GATED
// form) and up to 4 rows of x; a lane holds 16 bytes of each weight row per step,
// the group's warps take turns along k.  Sums are packed pairs of floats (even
// and odd k), joined over the lanes, then over the warps, in a fixed order.
//
// Two to 16 rows of aligned 16-bit operands, tensor cores by mma.sync: each weight
// meets so few rows that the tcgen05 kernel's tiles of 128 would be empty, and its
// weights would go by way of shared memory; see mma_rows_kernel.
//
// Measured on 4096 x 4096 bfloat16 in the L2, us: 1 row 5.1 (6.6 TB/s) on the FP32
// units; 4 rows 10.1 on them and 5.4 by mma.sync, 8 rows 5.7, 16 rows 7.1; the
// tcgen05 kernel and its join 12.8 at 17 rows.
#include <algorithm>

#include "layers_elem.cuh"
#include "layers_tc.h"

namespace vqc {
namespace layers {

namespace {

constexpr int kWeights = 4;    // weight rows of a group
constexpr int kWarps = 8;

struct RowsArgs {
    const void *x, *w0, *w1;
    Finish f;
    int64_t ld_x, ld_w, k;
    int kw;
};

// VEC elements as they lie in memory, and as pairs of floats
template <int VEC> struct Raw {
    uint32_t w[VEC == 1 ? 1 : 4];
};
template <typename T, int VEC> __device__ __forceinline__ Raw<VEC> load_raw(const T* q, bool in) {
    Raw<VEC> r{};
    if (!in) return r;
    if constexpr (VEC > 1) {
        const uint4 v = *reinterpret_cast<const uint4*>(q);
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else if constexpr (sizeof(T) == 4) {
        r.w[0] = __float_as_uint(*q);
    } else {
        r.w[0] = *reinterpret_cast<const uint16_t*>(q);
    }
    return r;
}
template <int VEC> struct Pairs {
    static constexpr int N = VEC < 2 ? 1 : VEC / 2;
    float2 p[N];
};
template <typename T, int VEC> __device__ __forceinline__ Pairs<VEC> pairs(const Raw<VEC>& v) {
    Pairs<VEC> r;
    if constexpr (sizeof(T) == 4) {
        if constexpr (VEC == 1) {
            r.p[0] = make_float2(__uint_as_float(v.w[0]), 0.f);
        } else {
            r.p[0] = make_float2(__uint_as_float(v.w[0]), __uint_as_float(v.w[1]));
            r.p[1] = make_float2(__uint_as_float(v.w[2]), __uint_as_float(v.w[3]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < Pairs<VEC>::N; ++i) r.p[i] = unpack2<T>(v.w[i]);      // one element: its pair's other is 0
    }
    return r;
}

template <typename T, int VEC, int R, bool GATE>
__global__ void __launch_bounds__(kWarps * 32) rows_kernel(const __grid_constant__ RowsArgs A) {
    constexpr int C = GATE ? kWeights / 2 : kWeights;   // output columns of a group
    __shared__ float sums[kWarps][R * kWeights];
    stream_order();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kw = A.kw;
    const int64_t group = (int64_t)blockIdx.x * (kWarps / kw) + warp / kw, c0 = group * C;
    const int64_t n = A.f.n;
    const int first = (int)blockIdx.y * R, m = (int)A.f.m - first;      // rows first, ..., first + R - 1
    const T* w[kWeights];
#pragma unroll
    for (int i = 0; i < kWeights; ++i) {
        const int64_t c = min(c0 + i % C, n - 1);
        w[i] = static_cast<const T*>(GATE && i >= C ? A.w1 : A.w0) + c * A.ld_w;
    }
    const T* x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = static_cast<const T*>(A.x) + (first + min(r, m - 1)) * A.ld_x;
    float2 acc[R][kWeights];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < kWeights; ++i) acc[r][i] = make_float2(0.f, 0.f);
    if (c0 < n) {
        // the weights of U steps are asked for before the first is used
        constexpr int U = VEC == 1 ? 8 : R == 1 && sizeof(T) == 2 ? 4 : 2;
        const int64_t step = (int64_t)kw * 32 * VEC;
        for (int64_t k0 = (int64_t)(warp % kw) * 32 * VEC; k0 < A.k; k0 += U * step) {
            Raw<VEC> rw[U][kWeights];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = k0 + u * step + lane * VEC;
#pragma unroll
                for (int i = 0; i < kWeights; ++i) rw[u][i] = load_raw<T, VEC>(w[i] + k, k < A.k);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = k0 + u * step + lane * VEC;
                Pairs<VEC> pw[kWeights];
#pragma unroll
                for (int i = 0; i < kWeights; ++i) pw[i] = pairs<T, VEC>(rw[u][i]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const Pairs<VEC> px = pairs<T, VEC>(load_raw<T, VEC>(x[r] + k, k < A.k));
#pragma unroll
                    for (int i = 0; i < kWeights; ++i)
#pragma unroll
                        for (int e = 0; e < Pairs<VEC>::N; ++e) acc[r][i] = fma2(pw[i].p[e], px.p[e], acc[r][i]);
                }
            }
        }
    }
    let_next();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < kWeights; ++i) {
            float s = acc[r][i].x + acc[r][i].y;
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
            if (lane == 0) sums[warp][r * kWeights + i] = s;
        }
    __syncthreads();
    // one thread per output of the CTA's groups
    const int groups = kWarps / kw;
    for (int e = threadIdx.x; e < groups * R * C; e += kWarps * 32) {
        const int g = e / (R * C), r = e / C % R, i = e % C;
        const int64_t c = ((int64_t)blockIdx.x * groups + g) * C + i;
        if (r >= m || c >= n) continue;
        float v0 = 0.f, v1 = 0.f;
        for (int q = 0; q < kw; ++q) {
            v0 += sums[g * kw + q][r * kWeights + i];
            if (GATE) v1 += sums[g * kw + q][r * kWeights + C + i];
        }
        finish_one(A.f, 0, first + r, c, v0, v1);
    }
}

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2], __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2], __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// Steps whose loads a warp has in flight: many warps with one each of a gate's weights, fewer warps
// with four of a plain product's.  From HBM, us: 4 x 2048 to 2 x 5632 9.7 so and 10.9 the
// other way, 4 x 4096 to 2 x 11008 31 and 32; 4 x 4096 to 4096 7.7 and 10.0, 4 x 8192 to 8192 21.7
// (6.2 TB/s) and 24.0.
constexpr int steps_ahead(bool gate) { return gate ? 1 : 4; }

// A group of KW warps takes 16 rows of weights (8 of each in GATED form: then both
// factors of an output are in one lane) and NB * 8 rows of x.  Lane 4 g + q loads 32
// bytes, k = 16 q + [0, 16) of the step's 64, of weight rows g and g + 8 (a whole line
// of each row by four lanes) and of rows g (and g + 8) of x; a contraction may take its
// elements in any order, so these are the operands of four products of depth 16 as they
// are: no shared memory, no shuffles.  The tensor cores cut the low bits of a running sum at
// every product (all terms positive, depth 8192 in one sum: 4.7e-5 of it), so a step's
// four products are a sum of their own and the steps are added as floats.
template <typename T, int NB, bool GATE>
__global__ void __launch_bounds__(kWarps * 32, GATE ? 6 - NB : 2) mma_rows_kernel(const __grid_constant__ RowsArgs A) {
    constexpr int C = GATE ? 8 : 16, U = steps_ahead(GATE);      // columns of a group, steps in flight
    __shared__ float sums[kWarps][NB * 4][33];
    stream_order();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kw = A.kw, g = lane >> 2;
    const int64_t group = (int64_t)blockIdx.x * (kWarps / kw) + warp / kw, c0 = group * C, n = A.f.n;
    const int m = (int)A.f.m;
    const int64_t second = GATE ? c0 + g : c0 + g + 8;
    const T* w0 = static_cast<const T*>(A.w0) + min(c0 + g, n - 1) * A.ld_w;
    const T* w1 = static_cast<const T*>(GATE ? A.w1 : A.w0) + min(second, n - 1) * A.ld_w;
    const T* x[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = static_cast<const T*>(A.x) + min(8 * b + g, m - 1) * A.ld_x;
    float acc[NB][4] = {};
    if (c0 < n) {
        const int64_t step = 64 * kw;
        for (int64_t k0 = 64 * (warp % kw); k0 < A.k; k0 += U * step) {
            uint4 a[U][2], b[U][2], y[U][NB][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t k = k0 + u * step + 16 * (lane & 3) + 8 * h;
                    const bool in = k < A.k;
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    a[u][h] = in ? *reinterpret_cast<const uint4*>(w0 + k) : zero;
                    b[u][h] = in ? *reinterpret_cast<const uint4*>(w1 + k) : zero;
#pragma unroll
                    for (int i = 0; i < NB; ++i) y[u][i][h] = in ? *reinterpret_cast<const uint4*>(x[i] + k) : zero;
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float part[NB][4] = {};      // a step's sum
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        const uint4 &p = a[u][h], &q = b[u][h], &z = y[u][i][h];
                        const uint32_t a0[4] = {p.x, q.x, p.y, q.y}, a1[4] = {p.z, q.z, p.w, q.w};
                        const uint32_t y0[2] = {z.x, z.y}, y1[2] = {z.z, z.w};
                        mma_16816(part[i], a0, y0, T());
                        mma_16816(part[i], a1, y1, T());
                    }
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][e] += part[i][e];
            }
        }
    }
    let_next();
    // sums of weight rows g (0, 1) and g + 8 (2, 3) with rows 2 q and 2 q + 1 of x
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[warp][4 * i + e][lane] = acc[i][e];
    __syncthreads();
    const int groups = kWarps / kw;
    for (int e = threadIdx.x; e < groups * 8 * NB * C; e += kWarps * 32) {
        const int q = e / (8 * NB * C), r = e / C % (8 * NB), i = e % C;       // group, row of x, column
        const int64_t c = ((int64_t)blockIdx.x * groups + q) * C + i;
        if (r >= m || c >= n) continue;
        const int at = 4 * (r / 8) + (r & 1), from = 4 * (i & 7) + (r % 8) / 2;
        float v0 = 0.f, v1 = 0.f;
        for (int k = 0; k < kw; ++k) {
            v0 += sums[q * kw + k][at + (!GATE && i >= 8 ? 2 : 0)][from];
            if (GATE) v1 += sums[q * kw + k][at + 2][from];
        }
        finish_one(A.f, 0, r, c, v0, v1);
    }
}

template <typename T> const void* mma_kernel_of(int64_t m, bool gate) {
    if (m <= 8) return gate ? (const void*)mma_rows_kernel<T, 1, true> : (const void*)mma_rows_kernel<T, 1, false>;
    return gate ? (const void*)mma_rows_kernel<T, 2, true> : (const void*)mma_rows_kernel<T, 2, false>;
}

template <typename T, int VEC, bool GATE> const void* kernel_of(int64_t m) {
    return m == 1   ? (const void*)rows_kernel<T, VEC, 1, GATE>
           : m == 2 ? (const void*)rows_kernel<T, VEC, 2, GATE>
                    : (const void*)rows_kernel<T, VEC, 4, GATE>;
}
template <typename T> const void* kernel_as(int64_t m, bool vec, bool gate) {
    constexpr int V = 16 / sizeof(T);
    if (vec) return gate ? kernel_of<T, V, true>(m) : kernel_of<T, V, false>(m);
    return gate ? kernel_of<T, 1, true>(m) : kernel_of<T, 1, false>(m);
}

// operands whose rows hold whole packs of 16 bytes on 16-byte boundaries
bool packed(const Product& p) {
    const int64_t per16 = 16 / (int64_t)elem_size(p.f.dtype);
    return p.k % per16 == 0 && p.a[0].ld % per16 == 0 && p.b[0].ld % per16 == 0;
}

}  // namespace

bool rows_takes(const Product& p, bool aligned) {
    if (p.m < 1 || p.k <= 0 || (p.form != PLAIN && p.form != GATED) || p.a[0].k_outer || p.b[0].k_outer) return false;
    return p.m <= 4 || (p.m <= 16 && (p.f.dtype == VQC_F32 || (aligned && packed(p))));
}

vqc_status rows_run(const Product& p, bool aligned, cudaStream_t s) {
    RowsArgs a{};
    const bool gate = p.form == GATED, vec = aligned && packed(p), mma = vec && p.m > 1 && p.f.dtype != VQC_F32;
    a.x = p.a[0].p;
    a.w0 = p.b[0].p;
    a.w1 = gate ? p.b[1].p : nullptr;
    a.f = p.f;
    a.ld_x = p.a[0].ld;
    a.ld_w = p.b[0].ld;
    a.k = p.k;
    // Warps per group: until there are enough per SM, with a few steps each at least
    const int64_t weights = mma ? 16 : kWeights, groups = ceil_div(p.n, gate ? weights / 2 : weights);
    const int64_t step = mma ? 64 * steps_ahead(gate) : 32 * (vec ? 16 / (int64_t)elem_size(p.f.dtype) : 1);
    int kw = 1;
    const int64_t enough = (mma ? (gate ? 32LL : 8LL) : 24LL) * sm_count(), rounds = mma ? (gate ? 2 : 1) : 4;
    while (kw < kWarps && groups * kw < enough && p.k >= rounds * step * kw) kw *= 2;
    a.kw = kw;
    const int64_t grid = ceil_div(groups, kWarps / kw);
    if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "too many columns");
    void* args[] = {&a};
    const void* fn = mma                        ? (p.f.dtype == VQC_BF16 ? mma_kernel_of<__nv_bfloat16>(p.m, gate) : mma_kernel_of<__half>(p.m, gate))
                     : p.f.dtype == VQC_F32     ? kernel_as<float>(p.m, vec, gate)
                     : p.f.dtype == VQC_BF16    ? kernel_as<__nv_bfloat16>(p.m, vec, gate)
                                                : kernel_as<__half>(p.m, vec, gate);
    const cudaError_t e = launch(fn, dim3((unsigned)grid, mma ? 1 : (unsigned)ceil_div(p.m, 4)), kWarps * 32, args, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "product of few rows launch");
}

}  // namespace layers
}  // namespace vqc
