// layer_norm.cu -- layer norm over the columns of each row, forward and backward.
//
// A row stays in registers between its statistics and its result: x is read
// once (forward), x and grad_y once (backward), each result written once, which
// is all that bounds these kernels.  Statistics in float: the mean first, then
// the sum of squared differences from it, so that rows with a large mean lose
// nothing.  The backward's column sums (gradients of weight and bias) stay in
// registers over all rows of a CTA: a thread owns the same columns of every
// row; the CTAs' sums are joined by sum_run in a fixed order.
//
// Rows longer than the registers hold take kernels that read their row again.
#include <algorithm>

#include "layers_elem.cuh"

namespace vqc {
namespace layers {

namespace {

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// Sums over the WARPS warps of a row, the same value in every thread: over the lanes, then
// (through `buf`) over the warps by every warp for itself.  Two buffers are used in
// turn, so that one barrier per sum is enough.
template <int WARPS> __device__ __forceinline__ float row_sum(float s, float* buf) {
    s = warp_sum(s);
    if (WARPS == 1) return s;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s;
    __syncthreads();
    s = buf[threadIdx.x & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    return s;
}
template <int WARPS> __device__ __forceinline__ float2 row_sum(float s, float t, float2* buf) {
    s = warp_sum(s);
    t = warp_sum(t);
    if (WARPS == 1) return make_float2(s, t);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = make_float2(s, t);
    __syncthreads();
    const float2 p = buf[threadIdx.x & (WARPS - 1)];
    s = p.x;
    t = p.y;
#pragma unroll
    for (int o = WARPS / 2; o; o >>= 1) {
        s += __shfl_xor_sync(~0u, s, o);
        t += __shfl_xor_sync(~0u, t, o);
    }
    return make_float2(s, t);
}

struct NormArgs {
    const void *x, *weight, *bias, *gy;
    void *y, *gx;
    const float* stats_in;
    float* stats;
    float* part;         // [2][CTAs][cols] column sums of the backward, or NULL
    int64_t rows, cols, ld_x, ld_gy;
    float eps;
};

// (the type of unpack2 where T is a 16-bit type)
template <typename T> struct Half {
    using type = T;
};
template <> struct Half<float> {
    using type = __half;
};

// VEC neighbouring elements as they lie in memory: one element, or 16 bytes
template <typename T, int VEC> struct alignas(VEC == 1 ? 4 : 16) Pack {
    uint32_t w[VEC == 1 ? 1 : 4];
};
template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> load_pack(const T* p) {
    Pack<T, VEC> r;
    if constexpr (VEC > 1) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        r.w[0] = q.x; r.w[1] = q.y; r.w[2] = q.z; r.w[3] = q.w;
    } else if constexpr (sizeof(T) == 4) {
        r.w[0] = __float_as_uint(*p);
    } else {
        r.w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    return r;
}
// the same as floats, in pairs (one element: the first of a pair)
template <int VEC> struct Lanes {
    static constexpr int N = VEC == 1 ? 1 : VEC / 2;
    float2 p[N];
};
template <typename T, int VEC> __device__ __forceinline__ void unpack(const Pack<T, VEC>& p, Lanes<VEC>& v) {
    if constexpr (VEC == 1) {
        v.p[0] = make_float2(sizeof(T) == 4 ? __uint_as_float(p.w[0]) : unpack2<typename Half<T>::type>(p.w[0]).x, 0.f);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) v.p[e] = make_float2(__uint_as_float(p.w[2 * e]), __uint_as_float(p.w[2 * e + 1]));
    } else {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) v.p[e] = unpack2<T>(p.w[e]);
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store_pack(T* p, const Lanes<VEC>& v) {
    if constexpr (VEC == 1) *p = from_f<T>(v.p[0].x);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
    else
        *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v.p[0].x, v.p[0].y), pack2<T>(v.p[1].x, v.p[1].y), pack2<T>(v.p[2].x, v.p[2].y),
                                                  pack2<T>(v.p[3].x, v.p[3].y));
}
template <typename T, int VEC> __device__ __forceinline__ void load_param(const void* p, int c, float other, Lanes<VEC>& v) {
    if (p) {
        unpack<T, VEC>(load_pack<T, VEC>(static_cast<const T*>(p) + c), v);
    } else {
#pragma unroll
        for (int e = 0; e < Lanes<VEC>::N; ++e) v.p[e] = make_float2(other, other);
    }
}

// WARPS warps per row, NV packs of VEC elements per thread: pack i of thread t holds the
// columns (i * threads + t) * VEC + [0, VEC).  With one warp per row a CTA has 8 rows.
template <int VEC, int WARPS> struct Row {
    static constexpr int kThreads = WARPS * 32, kCta = WARPS == 1 ? 256 : kThreads;
    static __device__ __forceinline__ int column(int i) {
        return (i * kThreads + (int)(WARPS == 1 ? threadIdx.x & 31 : threadIdx.x)) * VEC;
    }
    static __device__ __forceinline__ int64_t first() { return WARPS == 1 ? blockIdx.x * 8ll + (threadIdx.x >> 5) : blockIdx.x; }
    static __device__ __forceinline__ int64_t step() { return WARPS == 1 ? gridDim.x * 8ll : gridDim.x; }
};

// A thread's packs of row r; zeros beyond the columns, nothing beyond the rows.
template <typename T, int VEC, int WARPS, int NV>
__device__ __forceinline__ void load_row(const NormArgs& A, const void* p, int64_t ld, int64_t r, Pack<T, VEC> (&v)[NV]) {
    using R = Row<VEC, WARPS>;
    if (r >= A.rows) return;
    const T* x = static_cast<const T*>(p) + r * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        v[i] = Pack<T, VEC>{};
        if (R::column(i) < (int)A.cols) v[i] = load_pack<T, VEC>(x + R::column(i));
    }
}

// 8192 x 4096 bfloat16: 27.5 us (4.9 TB/s; 8192 x 2048, half in the L2: 6.3). Instructions count here as
// much as bytes, so elements are converted once and kept as floats.
template <typename T, int VEC, int WARPS, int NV>
__global__ void __launch_bounds__(Row<VEC, WARPS>::kCta, (VEC * NV <= 16 || WARPS == 16 ? 1024 : 768) / Row<VEC, WARPS>::kCta)
norm_forward_kernel(const __grid_constant__ NormArgs A) {
    using R = Row<VEC, WARPS>;
    __shared__ float buf[2][WARPS];
    stream_order();
    const int cols = (int)A.cols;
    const float inv = 1.f / (float)cols;
    for (int64_t r = R::first(); r < A.rows; r += R::step()) {
        Pack<T, VEC> raw[NV];
        load_row<T, VEC, WARPS, NV>(A, A.x, A.ld_x, r, raw);
        Lanes<VEC> v[NV];
        float2 s = make_float2(0.f, 0.f), q = s;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            unpack<T, VEC>(raw[i], v[i]);
#pragma unroll
            for (int e = 0; e < Lanes<VEC>::N; ++e) s = add2(s, v[i].p[e]);
        }
        const float mean = row_sum<WARPS>(s.x + s.y, buf[0]) * inv;
        const float2 minus = make_float2(-mean, VEC == 1 ? 0.f : -mean);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (R::column(i) < cols)
#pragma unroll
                for (int e = 0; e < Lanes<VEC>::N; ++e) {
                    v[i].p[e] = add2(v[i].p[e], minus);
                    q = fma2(v[i].p[e], v[i].p[e], q);
                }
        const float rstd = rsqrtf(row_sum<WARPS>(q.x + q.y, buf[1]) * inv + A.eps);
        if (A.stats && R::column(0) == 0) *reinterpret_cast<float2*>(A.stats + 2 * r) = make_float2(mean, rstd);
        T* y = static_cast<T*>(A.y) + r * cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = R::column(i);
            if (c >= cols) continue;
            Lanes<VEC> w, b;
            load_param<T, VEC>(A.weight, c, 1.f, w);
            load_param<T, VEC>(A.bias, c, 0.f, b);
#pragma unroll
            for (int e = 0; e < Lanes<VEC>::N; ++e) v[i].p[e] = fma2(mul2(v[i].p[e], make_float2(rstd, rstd)), w.p[e], b.p[e]);
            store_pack<T, VEC>(y + c, v[i]);
        }
    }
}

// Loads run a row ahead in registers, so that they are in flight during the sums of the row
// before (copies ahead into shared memory, four rows, were slower: 48 against 45 us at 8192 x 4096
// bfloat16).
template <typename T, int VEC, int WARPS, int NV>
__global__ void __launch_bounds__(Row<VEC, WARPS>::kCta) norm_backward_kernel(const __grid_constant__ NormArgs A) {
    using R = Row<VEC, WARPS>;
    __shared__ float2 buf[2][WARPS];
    stream_order();
    const int cols = (int)A.cols;
    const float inv = 1.f / (float)cols;
    constexpr int N = Lanes<VEC>::N;
    float2 gw[NV][N], gb[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) gw[i][e] = gb[i][e] = make_float2(0.f, 0.f);
    int turn = 0;
    Pack<T, VEC> nx[NV], ng[NV];
    load_row<T, VEC, WARPS, NV>(A, A.x, A.ld_x, R::first(), nx);
    load_row<T, VEC, WARPS, NV>(A, A.gy, A.ld_gy, R::first(), ng);
    auto stats_of = [&](int64_t r) { return r < A.rows ? *reinterpret_cast<const float2*>(A.stats_in + 2 * r) : make_float2(0.f, 0.f); };
    float2 s1 = stats_of(R::first()), s2 = stats_of(R::first() + R::step());     // two rows ahead as well
    for (int64_t r = R::first(); r < A.rows; r += R::step(), turn ^= 1) {
        const float2 st = s1;
        s1 = s2;
        s2 = stats_of(r + 2 * R::step());
        Lanes<VEC> h[NV], k[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            unpack<T, VEC>(nx[i], h[i]);
            unpack<T, VEC>(ng[i], k[i]);
        }
        load_row<T, VEC, WARPS, NV>(A, A.x, A.ld_x, r + R::step(), nx);
        load_row<T, VEC, WARPS, NV>(A, A.gy, A.ld_gy, r + R::step(), ng);
        const float2 minus = make_float2(-st.x, VEC == 1 ? 0.f : -st.x), scale = make_float2(st.y, st.y);
        float2 s = make_float2(0.f, 0.f), t = s;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (R::column(i) >= cols) continue;
            Lanes<VEC> w;
            load_param<T, VEC>(A.weight, R::column(i), 1.f, w);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                h[i].p[e] = mul2(add2(h[i].p[e], minus), scale);
                gw[i][e] = fma2(k[i].p[e], h[i].p[e], gw[i][e]);
                gb[i][e] = add2(gb[i][e], k[i].p[e]);
                k[i].p[e] = mul2(k[i].p[e], w.p[e]);
                s = add2(s, k[i].p[e]);
                t = fma2(k[i].p[e], h[i].p[e], t);
            }
        }
        if (!A.gx) continue;
        const float2 sum = row_sum<WARPS>(s.x + s.y, t.x + t.y, buf[turn]);
        const float2 ms = make_float2(-sum.x * inv, -sum.x * inv), mt = make_float2(-sum.y * inv, -sum.y * inv);
        T* gx = static_cast<T*>(A.gx) + r * cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (R::column(i) >= cols) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) k[i].p[e] = mul2(scale, fma2(h[i].p[e], mt, add2(k[i].p[e], ms)));
            store_pack<T, VEC>(gx + R::column(i), k[i]);
        }
    }
    let_next();
    if (!A.part) return;
    if constexpr (WARPS == 1) {   // the CTA's 8 rows' sums in the order of the warps
        __shared__ float sums[8][NV * VEC * 32];
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 p = which ? gb[i][e / 2] : gw[i][e / 2];
                    sums[threadIdx.x >> 5][R::column(i) + e] = e & 1 ? p.y : p.x;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += 256) {
                float a = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) a += sums[i][c];
                A.part[((int64_t)which * gridDim.x + blockIdx.x) * cols + c] = a;
            }
        }
    } else {
        float* pw = A.part + (int64_t)blockIdx.x * cols;
        float* pb = pw + (int64_t)gridDim.x * cols;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (R::column(i) < cols) {
                float *qw = pw + R::column(i), *qb = pb + R::column(i);
                if constexpr (VEC == 1) {
                    *qw = gw[i][0].x;
                    *qb = gb[i][0].x;
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; e += 4) {
                        *reinterpret_cast<float4*>(qw + e) = make_float4(gw[i][e / 2].x, gw[i][e / 2].y, gw[i][e / 2 + 1].x, gw[i][e / 2 + 1].y);
                        *reinterpret_cast<float4*>(qb + e) = make_float4(gb[i][e / 2].x, gb[i][e / 2].y, gb[i][e / 2 + 1].x, gb[i][e / 2 + 1].y);
                    }
                }
            }
    }
}

// ------------------------------------------------------------ rows beyond the registers

constexpr int kLong = 512;

template <typename T> __global__ void __launch_bounds__(kLong) norm_forward_long(const __grid_constant__ NormArgs A) {
    __shared__ float buf[2][kLong / 32];
    stream_order();
    for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(A.x) + r * A.ld_x;
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kLong) s += to_f(x[c]);
        const float mean = row_sum<kLong / 32>(s, buf[0]) / (float)A.cols;
        s = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kLong) {
            const float d = to_f(x[c]) - mean;
            s = fmaf(d, d, s);
        }
        const float rstd = rsqrtf(row_sum<kLong / 32>(s, buf[1]) / (float)A.cols + A.eps);
        if (A.stats && threadIdx.x == 0) *reinterpret_cast<float2*>(A.stats + 2 * r) = make_float2(mean, rstd);
        T* y = static_cast<T*>(A.y) + r * A.cols;
        for (int64_t c = threadIdx.x; c < A.cols; c += kLong) {
            const float w = A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f;
            const float b = A.bias ? to_f(static_cast<const T*>(A.bias)[c]) : 0.f;
            y[c] = from_f<T>(fmaf((to_f(x[c]) - mean) * rstd, w, b));
        }
    }
}

template <typename T> __global__ void __launch_bounds__(kLong) norm_backward_long(const __grid_constant__ NormArgs A) {
    __shared__ float2 buf[2][kLong / 32];
    stream_order();
    int turn = 0;
    for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x, turn ^= 1) {
        const T* x = static_cast<const T*>(A.x) + r * A.ld_x;
        const T* gy = static_cast<const T*>(A.gy) + r * A.ld_gy;
        const float mean = A.stats_in[2 * r], rstd = A.stats_in[2 * r + 1];
        float s = 0.f, t = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kLong) {
            const float g = to_f(gy[c]) * (A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f);
            s += g;
            t = fmaf(g, (to_f(x[c]) - mean) * rstd, t);
        }
        const float2 sum = row_sum<kLong / 32>(s, t, buf[turn]);
        s = sum.x / (float)A.cols;
        t = sum.y / (float)A.cols;
        T* gx = static_cast<T*>(A.gx) + r * A.cols;
        for (int64_t c = threadIdx.x; c < A.cols; c += kLong) {
            const float g = to_f(gy[c]) * (A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f);
            gx[c] = from_f<T>(rstd * (g - s - (to_f(x[c]) - mean) * rstd * t));
        }
    }
}

// Column sums over `per` rows: thread = column.
template <typename T> __global__ void __launch_bounds__(256) norm_columns_long(const __grid_constant__ NormArgs A, int64_t per) {
    stream_order();
    const int64_t across = (A.cols + 255) / 256, block = blockIdx.x / across, blocks = gridDim.x / across;
    const int64_t c = blockIdx.x % across * 256 + threadIdx.x;
    if (c >= A.cols) return;
    float s = 0.f, t = 0.f;
    const int64_t r1 = min(A.rows, (block + 1) * per);
#pragma unroll 4
    for (int64_t r = block * per; r < r1; ++r) {
        const float g = to_f(static_cast<const T*>(A.gy)[r * A.ld_gy + c]);
        s = fmaf(g, (to_f(static_cast<const T*>(A.x)[r * A.ld_x + c]) - A.stats_in[2 * r]) * A.stats_in[2 * r + 1], s);
        t += g;
    }
    A.part[block * A.cols + c] = s;
    A.part[(blocks + block) * A.cols + c] = t;
}

// ------------------------------------------------------------ choice and launch

// Threads per row so that a thread holds 8 or 16 elements (backward; as many sums
// twice) and up to 32 (forward); rows beyond 16 warps of these are `long`.
constexpr int64_t kMostForward = 16384, kMostBackward = 8192;

int64_t row_ctas(int warps, int64_t rows, int64_t most) {
    const int64_t n = warps == 1 ? ceil_div(rows, 8) : rows;
    return std::max<int64_t>(1, std::min<int64_t>(n, most));
}

struct Plan {
    const void* fn;
    int warps, threads;
};
template <typename T, int VEC, int WARPS, int NV> Plan forward_plan() {
    return {(const void*)norm_forward_kernel<T, VEC, WARPS, NV>, WARPS, Row<VEC, WARPS>::kCta};
}
template <typename T, int VEC, int WARPS, int NV> Plan backward_plan() {
    return {(const void*)norm_backward_kernel<T, VEC, WARPS, NV>, WARPS, Row<VEC, WARPS>::kCta};
}
// E: elements per thread and step of the ladder
template <typename T, int VEC> Plan forward_choice(int64_t cols) {
    constexpr int N8 = 8 / VEC, N16 = 16 / VEC, N32 = 32 / VEC;
    if constexpr (VEC == 1) {      // single elements: more threads, fewer loads each
        if (cols <= 256) return forward_plan<T, VEC, 1, N8>();
        if (cols <= 512) return forward_plan<T, VEC, 2, N8>();
        if (cols <= 1024) return forward_plan<T, VEC, 4, N8>();
        if (cols <= 2048) return forward_plan<T, VEC, 8, N8>();
        if (cols <= 4096) return forward_plan<T, VEC, 16, N8>();
        if (cols <= 8192) return forward_plan<T, VEC, 16, N16>();
        return forward_plan<T, VEC, 16, N32>();
    } else {
        if (cols <= 256) return forward_plan<T, VEC, 1, N8>();
        if (cols <= 512) return forward_plan<T, VEC, 1, N16>();
        if (cols <= 1024) return forward_plan<T, VEC, 1, N32>();
        if (cols <= 2048) return forward_plan<T, VEC, 2, N32>();
        if (cols <= 4096) return forward_plan<T, VEC, 4, N32>();
        if (cols <= 8192) return forward_plan<T, VEC, 8, N32>();
        return forward_plan<T, VEC, 16, N32>();
    }
}
template <typename T, int VEC> Plan backward_choice(int64_t cols) {
    constexpr int N8 = 8 / VEC, N16 = 16 / VEC;
    if (cols <= 256) return backward_plan<T, VEC, 1, N8>();
    if constexpr (VEC == 1) {
        if (cols <= 512) return backward_plan<T, VEC, 2, N8>();
        if (cols <= 1024) return backward_plan<T, VEC, 4, N8>();
        if (cols <= 2048) return backward_plan<T, VEC, 8, N8>();
        if (cols <= 4096) return backward_plan<T, VEC, 16, N8>();
    } else {
        if (cols <= 512) return backward_plan<T, VEC, 1, N16>();
        if (cols <= 1024) return backward_plan<T, VEC, 2, N16>();
        if (cols <= 2048) return backward_plan<T, VEC, 4, N16>();
        if (cols <= 4096) return backward_plan<T, VEC, 8, N16>();
    }
    return backward_plan<T, VEC, 16, N16>();
}
template <typename T> Plan choose_plan(bool forward, int64_t cols, bool vec) {
    constexpr int V = 16 / sizeof(T);
    if (forward) return vec ? forward_choice<T, V>(cols) : forward_choice<T, 1>(cols);
    return vec ? backward_choice<T, V>(cols) : backward_choice<T, 1>(cols);
}
Plan choose_plan(int dtype, bool forward, int64_t cols, bool vec) {
    return dtype == VQC_F32    ? choose_plan<float>(forward, cols, vec)
           : dtype == VQC_BF16 ? choose_plan<__nv_bfloat16>(forward, cols, vec)
                               : choose_plan<__half>(forward, cols, vec);
}
template <typename T> const void* long_kernel(int which) {
    return which == 0 ? (const void*)norm_forward_long<T>
           : which == 1 ? (const void*)norm_backward_long<T> : (const void*)norm_columns_long<T>;
}
const void* long_kernel(int dtype, int which) {
    return dtype == VQC_F32 ? long_kernel<float>(which) : dtype == VQC_BF16 ? long_kernel<__nv_bfloat16>(which) : long_kernel<__half>(which);
}

// CTAs of the backward, each with its column sums: few, since the sums are written and read
// again, and as many as their registers (about 100 a thread) allow at one time.
int64_t backward_ctas(int warps, int64_t cols, int64_t rows) {
    const int per_sm = cols <= 256 ? 4 : cols <= 512 ? 2 : cols <= 1024 ? 4 : cols <= 2048 ? 3 : cols <= 4096 ? 2 : 1;
    return row_ctas(warps, rows, (int64_t)sm_count() * per_sm);
}
constexpr int64_t kLongBlocks = 64;   // blocks of rows of norm_columns_long

// rows and vectors on 16-byte boundaries
bool packs(size_t e, int64_t cols, std::initializer_list<const void*> p, std::initializer_list<int64_t> strides) {
    if (cols * e % 16) return false;
    for (const void* q : p)
        if (!aligned_to(q, 16)) return false;
    for (int64_t s : strides)
        if (s * e % 16) return false;
    return true;
}

vqc_status launched(cudaError_t e) { return e == cudaSuccess ? VQC_OK : cuda_error(e, "layer norm launch"); }

}  // namespace
}  // namespace layers
}  // namespace vqc

using namespace vqc;
using namespace vqc::layers;

extern "C" {

vqc_status vqc_layer_norm_forward(vqc_real dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                                  const void* weight, const void* bias, double eps, void* y, float* stats, void* stream) {
    try {
        if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || rows < 0 || cols < 1 || cols > 0x7fffffff ||
            x_stride < cols || !(eps >= 0) || (rows > 0 && (!x || !y)))
            return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_forward: bad type, size, stride, eps or NULL pointer");
        const size_t e = elem_size(dtype);
        if (!aligned_to(x, e) || !aligned_to(weight, e) || !aligned_to(bias, e) || !aligned_to(y, 16) || !aligned_to(stats, 8))
            return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_forward: misaligned operand or output");
        if (rows == 0) return VQC_OK;
        NormArgs a{};
        a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.stats = stats;
        a.rows = rows; a.cols = cols; a.ld_x = x_stride; a.eps = (float)eps;
        void* args[] = {&a};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        if (cols > kMostForward)
            return launched(launch(long_kernel(dtype, 0), dim3((unsigned)std::min<int64_t>(rows, 4LL * sm_count())), kLong, args, s));
        const Plan p = choose_plan(dtype, true, cols, packs(e, cols, {x, weight, bias, y}, {x_stride}));
        return launched(launch(p.fn, dim3((unsigned)row_ctas(p.warps, rows, 0x7fffffff)), p.threads, args, s));
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

size_t vqc_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || cols > 0x7fffffff) return (size_t)-1;
    const int64_t blocks = cols > kMostBackward ? kLongBlocks : backward_ctas(2, cols, rows);     // a CTA with 8 rows has fewer
    return align256((size_t)2 * blocks * cols * 4);
}

vqc_status vqc_layer_norm_backward(vqc_real dtype, int64_t rows, int64_t cols, const void* grad_y, int64_t grad_y_stride,
                                   const void* x, int64_t x_stride, const void* weight, const float* stats, void* grad_x,
                                   void* grad_weight, void* grad_bias, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    try {
        if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || rows < 0 || cols < 1 || cols > 0x7fffffff ||
            x_stride < cols || grad_y_stride < cols || (rows > 0 && (!x || !grad_y || !stats)))
            return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_backward: bad type, size, stride or NULL pointer");
        const size_t e = elem_size(dtype);
        if (!aligned_to(x, e) || !aligned_to(grad_y, e) || !aligned_to(weight, e) || !aligned_to(grad_x, 16) ||
            !aligned_to(grad_weight, e) || !aligned_to(grad_bias, e) || !aligned_to(stats, 8) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_backward: misaligned operand, output or workspace");
        const bool columns = grad_weight || grad_bias;
        if (columns && (!workspace || workspace_bytes < vqc_layer_norm_workspace_bytes(rows, cols)))
            return set_error(VQC_ERR_WORKSPACE, "vqc_layer_norm_backward: workspace too small");
        if (!columns && (!grad_x || rows == 0)) return VQC_OK;
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        NormArgs a{};
        a.x = x; a.weight = weight; a.gy = grad_y; a.gx = grad_x; a.stats_in = stats;
        a.rows = rows; a.cols = cols; a.ld_x = x_stride; a.ld_gy = grad_y_stride;
        a.part = columns ? static_cast<float*>(workspace) : nullptr;
        int64_t blocks = 0;
        if (rows > 0 && cols > kMostBackward) {
            int64_t per = ceil_div(rows, kLongBlocks);
            void* args[] = {&a, &per};
            if (grad_x) {
                const cudaError_t err = launch(long_kernel(dtype, 1), dim3((unsigned)std::min<int64_t>(rows, 4LL * sm_count())), kLong, args, s);
                if (err != cudaSuccess) return launched(err);
            }
            if (columns) {
                blocks = ceil_div(rows, per);
                const int64_t grid = blocks * ceil_div(cols, 256);
                if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_backward: too many columns");
                const cudaError_t err = launch(long_kernel(dtype, 2), dim3((unsigned)grid), 256, args, s);
                if (err != cudaSuccess) return launched(err);
            }
        } else if (rows > 0) {
            const Plan p = choose_plan(dtype, false, cols, packs(e, cols, {x, weight, grad_y, grad_x}, {x_stride, grad_y_stride}));
            blocks = backward_ctas(p.warps, cols, rows);
            void* args[] = {&a};
            const cudaError_t err = launch(p.fn, dim3((unsigned)blocks), p.threads, args, s);
            if (err != cudaSuccess) return launched(err);
        }
        return columns ? sum_run(a.part, blocks, cols, cols, blocks * cols, grad_weight, grad_bias, dtype, s) : VQC_OK;
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
