// layer_norm.cu -- layer norm over the columns of each row, forward and backward.
//
// Statistics in float: the mean first, then the sum of squared differences from
// it, so that rows with a large mean lose nothing.
#include <algorithm>

#include "layers_elem.cuh"

namespace vqc {
namespace layers {

vqc_status sum_run(const float* part, int64_t count, int64_t n, void* out0, void* out1, int dtype, cudaStream_t s);

namespace {

constexpr int kNormThreads = 256;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// sum over the CTA, the same value in every thread
__device__ __forceinline__ float cta_sum(float v, float* buf) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < kNormThreads / 32; ++i) v += buf[i];
    return v;
}

struct NormArgs {
    const void *x, *weight, *bias, *gy;
    void *y, *gx;
    const float* stats_in;
    float* stats;
    float* part;         // [2][CTAs][cols] column sums of the backward
    int64_t rows, cols, ld_x, ld_gy;
    float eps;
};

template <typename T> __global__ void __launch_bounds__(kNormThreads) norm_forward_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float buf[kNormThreads / 32];
    for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(A.x) + r * A.ld_x;
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kNormThreads) s += to_f(x[c]);
        const float mean = cta_sum(s, buf) / (float)A.cols;
        s = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kNormThreads) {
            const float d = to_f(x[c]) - mean;
            s = fmaf(d, d, s);
        }
        const float rstd = 1.f / sqrtf(cta_sum(s, buf) / (float)A.cols + A.eps);
        if (A.stats && threadIdx.x == 0) {
            A.stats[2 * r] = mean;
            A.stats[2 * r + 1] = rstd;
        }
        T* y = static_cast<T*>(A.y) + r * A.cols;
        for (int64_t c = threadIdx.x; c < A.cols; c += kNormThreads) {
            const float w = A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f;
            const float b = A.bias ? to_f(static_cast<const T*>(A.bias)[c]) : 0.f;
            y[c] = from_f<T>(fmaf((to_f(x[c]) - mean) * rstd, w, b));
        }
    }
}

template <typename T> __global__ void __launch_bounds__(kNormThreads) norm_backward_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float buf[kNormThreads / 32];
    for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(A.x) + r * A.ld_x;
        const T* gy = static_cast<const T*>(A.gy) + r * A.ld_gy;
        const float mean = A.stats_in[2 * r], rstd = A.stats_in[2 * r + 1];
        float s = 0.f, t = 0.f;
        for (int64_t c = threadIdx.x; c < A.cols; c += kNormThreads) {
            const float g = to_f(gy[c]) * (A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f);
            s += g;
            t = fmaf(g, (to_f(x[c]) - mean) * rstd, t);
        }
        s = cta_sum(s, buf) / (float)A.cols;
        t = cta_sum(t, buf) / (float)A.cols;
        if (!A.gx) continue;
        T* gx = static_cast<T*>(A.gx) + r * A.cols;
        for (int64_t c = threadIdx.x; c < A.cols; c += kNormThreads) {
            const float g = to_f(gy[c]) * (A.weight ? to_f(static_cast<const T*>(A.weight)[c]) : 1.f);
            gx[c] = from_f<T>(rstd * (g - s - (to_f(x[c]) - mean) * rstd * t));
        }
    }
}

// Column sums over the rows of one CTA: thread = column.
template <typename T> __global__ void __launch_bounds__(kNormThreads) norm_columns_kernel(const __grid_constant__ NormArgs A, int64_t per) {
    const int64_t across = (A.cols + kNormThreads - 1) / kNormThreads, block = blockIdx.x / across, blocks = gridDim.x / across;
    const int64_t c = blockIdx.x % across * kNormThreads + threadIdx.x;
    if (c >= A.cols) return;
    float s = 0.f, t = 0.f;
    const int64_t r1 = min(A.rows, (block + 1) * per);
    for (int64_t r = block * per; r < r1; ++r) {
        const float g = to_f(static_cast<const T*>(A.gy)[r * A.ld_gy + c]);
        s = fmaf(g, (to_f(static_cast<const T*>(A.x)[r * A.ld_x + c]) - A.stats_in[2 * r]) * A.stats_in[2 * r + 1], s);
        t += g;
    }
    A.part[block * A.cols + c] = s;
    A.part[(blocks + block) * A.cols + c] = t;
}

template <typename T> cudaError_t launch(int which, NormArgs a, int grid, int64_t per, cudaStream_t s) {
    void* args[] = {&a, &per};
    const void* fn = which == 0 ? (const void*)norm_forward_kernel<T>
                     : which == 1 ? (const void*)norm_backward_kernel<T> : (const void*)norm_columns_kernel<T>;
    return cudaLaunchKernel(fn, dim3(grid), dim3(kNormThreads), args, 0, s);
}
cudaError_t launch_as(int dtype, int which, const NormArgs& a, int64_t grid, int64_t per, cudaStream_t s) {
    if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return dtype == VQC_F32    ? launch<float>(which, a, (int)grid, per, s)
           : dtype == VQC_BF16 ? launch<__nv_bfloat16>(which, a, (int)grid, per, s)
                               : launch<__half>(which, a, (int)grid, per, s);
}

constexpr int64_t kNormBlocks = 64;   // blocks of rows of the column sums

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
        const cudaError_t err = launch_as(dtype, 0, a, std::min<int64_t>(rows, 8LL * sm_count()), 0, static_cast<cudaStream_t>(stream));
        return err == cudaSuccess ? VQC_OK : cuda_error(err, "layer norm launch");
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

size_t vqc_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || cols > 0x7fffffff) return (size_t)-1;
    return align256((size_t)2 * kNormBlocks * cols * 4);
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
            !aligned_to(grad_weight, e) || !aligned_to(grad_bias, e) || !aligned_to(stats, 4) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, "vqc_layer_norm_backward: misaligned operand, output or workspace");
        const bool columns = grad_weight || grad_bias;
        if (columns && (!workspace || workspace_bytes < vqc_layer_norm_workspace_bytes(rows, cols)))
            return set_error(VQC_ERR_WORKSPACE, "vqc_layer_norm_backward: workspace too small");
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        NormArgs a{};
        a.x = x; a.weight = weight; a.gy = grad_y; a.gx = grad_x; a.stats_in = stats;
        a.rows = rows; a.cols = cols; a.ld_x = x_stride; a.ld_gy = grad_y_stride;
        a.part = static_cast<float*>(workspace);
        if (grad_x && rows > 0) {
            const cudaError_t err = launch_as(dtype, 1, a, std::min<int64_t>(rows, 8LL * sm_count()), 0, s);
            if (err != cudaSuccess) return cuda_error(err, "layer norm launch");
        }
        if (!columns) return VQC_OK;
        const int64_t per = ceil_div(rows, kNormBlocks), blocks = rows ? ceil_div(rows, per) : 0;
        if (blocks) {
            const cudaError_t err = launch_as(dtype, 2, a, blocks * ceil_div(cols, kNormThreads), per, s);
            if (err != cudaSuccess) return cuda_error(err, "layer norm launch");
        }
        if (grad_weight) {
            const vqc_status st = sum_run(a.part, blocks, cols, grad_weight, nullptr, dtype, s);
            if (st != VQC_OK) return st;
        }
        return grad_bias ? sum_run(a.part + blocks * cols, blocks, cols, grad_bias, nullptr, dtype, s) : VQC_OK;
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
