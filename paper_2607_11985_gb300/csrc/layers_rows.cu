// layers_rows.cu -- products with few rows (single tokens, small batches): the
// weights are all there is to read, so they stream through registers once.
//
// A group of KW warps takes four rows of weights (two of each in GATED form) and
// up to 4 rows of x; a lane holds 16 bytes of each weight row per step, the
// group's warps take turns along k.  Sums are packed pairs of floats (even and
// odd k), joined over the lanes, then over the warps, in a fixed order.
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

// VEC elements as pairs of floats
template <typename T, int VEC> struct Pairs {
    float2 p[VEC < 2 ? 1 : VEC / 2];
};
template <typename T, int VEC> __device__ __forceinline__ Pairs<T, VEC> load_pairs(const T* q, bool in) {
    Pairs<T, VEC> r;
    if constexpr (VEC == 1) {
        r.p[0] = make_float2(in ? to_f(*q) : 0.f, 0.f);
    } else {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (in) v = *reinterpret_cast<const uint4*>(q);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 4) {
            r.p[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
            r.p[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r.p[i] = unpack2<T>(w[i]);
        }
    }
    return r;
}

template <typename T, int VEC, int R, bool GATE>
__global__ void __launch_bounds__(kWarps * 32) rows_kernel(const __grid_constant__ RowsArgs A) {
    constexpr int C = GATE ? kWeights / 2 : kWeights;   // output columns of a group
    __shared__ float sums[kWarps][R * kWeights];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kw = A.kw;
    const int64_t group = (int64_t)blockIdx.x * (kWarps / kw) + warp / kw, c0 = group * C;
    const int64_t n = A.f.n;
    const int m = (int)A.f.m;
    const T* w[kWeights];
#pragma unroll
    for (int i = 0; i < kWeights; ++i) {
        const int64_t c = min(c0 + i % C, n - 1);
        w[i] = static_cast<const T*>(GATE && i >= C ? A.w1 : A.w0) + c * A.ld_w;
    }
    const T* x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = static_cast<const T*>(A.x) + min(r, m - 1) * A.ld_x;
    float2 acc[R][kWeights];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < kWeights; ++i) acc[r][i] = make_float2(0.f, 0.f);
    if (c0 < n) {
#pragma unroll(VEC == 1 ? 8 : 4)
        for (int64_t k = ((int64_t)(warp % kw) * 32 + lane) * VEC; k - lane * VEC < A.k; k += (int64_t)kw * 32 * VEC) {
            const bool in = k < A.k;
            Pairs<T, VEC> pw[kWeights];
#pragma unroll
            for (int i = 0; i < kWeights; ++i) pw[i] = load_pairs<T, VEC>(w[i] + k, in);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const Pairs<T, VEC> px = load_pairs<T, VEC>(x[r] + k, in);
#pragma unroll
                for (int i = 0; i < kWeights; ++i)
#pragma unroll
                    for (int e = 0; e < (VEC < 2 ? 1 : VEC / 2); ++e) acc[r][i] = fma2(pw[i].p[e], px.p[e], acc[r][i]);
            }
        }
    }
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
        finish_one(A.f, 0, r, c, v0, v1);
    }
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

}  // namespace

bool rows_takes(const Product& p) {
    return p.m >= 1 && p.m <= 4 && p.k > 0 && (p.form == PLAIN || p.form == GATED) && !p.a[0].k_outer && !p.b[0].k_outer;
}

vqc_status rows_run(const Product& p, cudaStream_t s) {
    RowsArgs a{};
    const bool gate = p.form == GATED;
    a.x = p.a[0].p;
    a.w0 = p.b[0].p;
    a.w1 = gate ? p.b[1].p : nullptr;
    a.f = p.f;
    a.ld_x = p.a[0].ld;
    a.ld_w = p.b[0].ld;
    a.k = p.k;
    const int64_t per16 = 16 / (int64_t)elem_size(p.f.dtype);
    const bool vec = p.k % per16 == 0 && a.ld_x % per16 == 0 && a.ld_w % per16 == 0 && aligned_to(a.x, 16) && aligned_to(a.w0, 16) && aligned_to(a.w1, 16);
    // Warps per group: until there are 24 warps per SM, with two steps each at least
    const int64_t groups = ceil_div(p.n, gate ? kWeights / 2 : kWeights), step = 32 * (vec ? per16 : 1);
    int kw = 1;
    while (kw < kWarps && groups * kw < 24LL * sm_count() && p.k >= 4 * step * kw) kw *= 2;
    a.kw = kw;
    const int64_t grid = ceil_div(groups, kWarps / kw);
    if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "too many columns");
    void* args[] = {&a};
    const void* fn = p.f.dtype == VQC_F32    ? kernel_as<float>(p.m, vec, gate)
                     : p.f.dtype == VQC_BF16 ? kernel_as<__nv_bfloat16>(p.m, vec, gate)
                                             : kernel_as<__half>(p.m, vec, gate);
    const cudaError_t e = cudaLaunchKernel(fn, dim3((unsigned)grid), dim3(kWarps * 32), args, 0, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "product of few rows launch");
}

}  // namespace layers
}  // namespace vqc
