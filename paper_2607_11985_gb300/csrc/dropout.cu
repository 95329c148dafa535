// dropout.cu -- dropout with a residual, from a counter-based generator.
//
// Element e of a tensor, counted in rows, is kept where word e % 4 of
//   Philox 4x32-10(counter = (e / 4, offset), key = seed)
// (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) is at least
// p 2^32, so that no mask is stored: the backward draws it again, in any order and launch shape.
//
// Bound by HBM (x and the residual once, y once) and nearly as much by the generator: 10 rounds of two 32 x 32 -> 64 bit
// products and two exclusive ors for four elements.  8192 x 4096 bfloat16: forward with a residual 32 us (6.3 TB/s),
// backward 30 us (4.4 TB/s: bound by the integer instructions).
#include <algorithm>
#include <cmath>

#include "layers_elem.cuh"

namespace vqc {
namespace layers {

namespace {

struct DropArgs {
    const void *x, *res;         // res may be NULL
    void* y;
    int64_t rows, cols, ld_x, ld_res;
    const uint64_t* state;       // (seed, offset) of the device, or NULL
    uint64_t seed, offset;
    uint32_t limit;              // words below it drop their element
    float scale;
    uint32_t key[20];            // of the rounds, from `seed`
};

// kState: the rounds' keys from a seed in memory; else as they come with the arguments, where they cost no instruction
// (two additions a round: 5 us more at 8192 x 4096).
template <bool kState> __device__ __forceinline__ uint4 philox(uint64_t block, uint64_t offset, uint64_t seed, const uint32_t* key) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        const uint32_t k0 = kState ? (uint32_t)seed + r * 0x9E3779B9u : key[2 * r], k1 = kState ? (uint32_t)(seed >> 32) + r * 0xBB67AE85u : key[2 * r + 1];
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ uint32_t word(const uint4& w, int i) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }

// What was dropped is zero whatever it held; one rounding of the sum.
__device__ __forceinline__ float dropped(float x, float res, uint32_t w, const DropArgs& A) {
    float y = res;
    if (w >= A.limit) y = fmaf(x, A.scale, res);
    return y;
}

// V elements (16 bytes) of a row at a time; a row holds whole packs, but for the last one of a single row.
// kFlat: one row.
template <typename T, bool kRes, bool kState, bool kFlat> __global__ void __launch_bounds__(256, 6) drop_kernel(const __grid_constant__ DropArgs A) {
    constexpr int V = 16 / sizeof(T);
    stream_order();
    const uint64_t seed = kState ? A.state[0] : A.seed, offset = A.offset + (kState ? A.state[1] : 0);
    const int64_t across = A.cols / V, packs = A.rows * across, step = (int64_t)gridDim.x * blockDim.x;
    const T *x = static_cast<const T*>(A.x), *res = static_cast<const T*>(A.res);
    T* y = static_cast<T*>(A.y);
    const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    auto at = [&](int64_t i, int64_t ld) {
        if (kFlat) return i * V;
        const int64_t r = packs >> 32 ? i / across : (int64_t)((uint32_t)i / (uint32_t)across);
        return r * ld + (i - r * across) * V;
    };
    for (int64_t i = first; i < packs; i += step) {
        const uint4 xv = *reinterpret_cast<const uint4*>(x + at(i, A.ld_x));
        const uint4 rv = kRes ? *reinterpret_cast<const uint4*>(res + at(i, A.ld_res)) : make_uint4(0, 0, 0, 0);
        const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, rw[4] = {rv.x, rv.y, rv.z, rv.w};
        uint32_t out[4];
#pragma unroll
        for (int b = 0; b < V / 4; ++b) {
            const uint4 w = philox<kState>((uint64_t)i * (V / 4) + b, offset, seed, A.key);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (sizeof(T) == 4) {
                    out[2 * h] = __float_as_uint(dropped(__uint_as_float(xw[2 * h]), __uint_as_float(rw[2 * h]), word(w, 2 * h), A));
                    out[2 * h + 1] = __float_as_uint(dropped(__uint_as_float(xw[2 * h + 1]), __uint_as_float(rw[2 * h + 1]), word(w, 2 * h + 1), A));
                } else {
                    const float2 a = unpack2<T>(xw[2 * b + h]), d = unpack2<T>(rw[2 * b + h]);
                    out[2 * b + h] = pack2<T>(dropped(a.x, d.x, word(w, 2 * h), A), dropped(a.y, d.y, word(w, 2 * h + 1), A));
                }
            }
        }
        *reinterpret_cast<uint4*>(y + i * V) = make_uint4(out[0], out[1], out[2], out[3]);
    }
    if (kFlat && first < A.cols - across * V) {
        const int64_t e = across * V + first;
        y[e] = from_f<T>(dropped(to_f(x[e]), kRes ? to_f(res[e]) : 0.f, word(philox<kState>((uint64_t)e / 4, offset, seed, A.key), (int)(e & 3)), A));
    }
}

// The same element by element, for rows that are not on 16-byte boundaries.
template <typename T> __global__ void __launch_bounds__(256) drop_any_kernel(const __grid_constant__ DropArgs A) {
    stream_order();
    const uint64_t seed = A.state ? A.state[0] : A.seed, offset = A.offset + (A.state ? A.state[1] : 0);
    const int64_t n = A.rows * A.cols, step = (int64_t)gridDim.x * blockDim.x;
    const T *x = static_cast<const T*>(A.x), *res = static_cast<const T*>(A.res);
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; 4 * i < n; i += step) {
        const uint4 w = philox<true>((uint64_t)i, offset, seed, nullptr);
        int64_t r = n >> 32 ? 4 * i / A.cols : (int64_t)((uint32_t)(4 * i) / (uint32_t)A.cols), c = 4 * i - r * A.cols;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (4 * i + j >= n) break;
            const float d = res ? to_f(res[r * A.ld_res + c]) : 0.f;
            static_cast<T*>(A.y)[4 * i + j] = from_f<T>(dropped(to_f(x[r * A.ld_x + c]), d, word(w, j), A));
            if (++c == A.cols) {
                c = 0;
                ++r;
            }
        }
    }
}

template <typename T, bool kRes, bool kState> const void* drop_fn(bool flat) {
    return flat ? (const void*)drop_kernel<T, kRes, kState, true> : (const void*)drop_kernel<T, kRes, kState, false>;
}
template <typename T> const void* drop_fn(bool packs, bool res, bool state, bool flat) {
    if (!packs) return (const void*)drop_any_kernel<T>;
    if (state) return res ? drop_fn<T, true, true>(flat) : drop_fn<T, false, true>(flat);
    return res ? drop_fn<T, true, false>(flat) : drop_fn<T, false, false>(flat);
}

vqc_status dropout(const char* call, int dtype, int64_t rows, int64_t cols, const void* x, int64_t ld_x, const void* res, int64_t ld_res,
                   double p, uint64_t seed, uint64_t offset, const uint64_t* state, void* y, void* stream) {
    if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || rows < 0 || cols < 1 || cols > 0x7fffffff ||
        (rows > 0 && rows > (int64_t(1) << 62) / cols) || ld_x < cols || (res && ld_res < cols) || !(p >= 0) || !(p < 1) || (rows > 0 && (!x || !y)))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": bad type, size, stride, probability or NULL pointer");
    const size_t e = elem_size(dtype);
    if (!aligned_to(x, e) || !aligned_to(res, e) || !aligned_to(y, 16) || !aligned_to(state, 8))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned operand or output");
    if (rows == 0) return VQC_OK;
    if (ld_x == cols && (!res || ld_res == cols)) {      // one row
        cols *= rows;
        ld_x = ld_res = cols;
        rows = 1;
    }
    DropArgs a{x, res, y, rows, cols, ld_x, ld_res, state, seed, offset, 0, (float)(1.0 / (1.0 - p)), {}};
    for (int r = 0; r < 10; ++r) {
        a.key[2 * r] = (uint32_t)seed + (uint32_t)r * 0x9E3779B9u;
        a.key[2 * r + 1] = (uint32_t)(seed >> 32) + (uint32_t)r * 0xBB67AE85u;
    }
    a.limit = (uint32_t)std::fmin(std::nearbyint(p * 4294967296.0), 4294967295.0);
    const int64_t v = 16 / (int64_t)e;
    const bool packs = aligned_to(x, 16) && aligned_to(res, 16) && (rows == 1 || (cols % v == 0 && ld_x % v == 0 && (!res || ld_res % v == 0)));
    const void* fn = dtype == VQC_F32 ? drop_fn<float>(packs, res, state, rows == 1) : dtype == VQC_BF16 ? drop_fn<__nv_bfloat16>(packs, res, state, rows == 1) : drop_fn<__half>(packs, res, state, rows == 1);
    const int64_t threads = ceil_div(rows * cols, packs ? v : 4);
    void* args[] = {&a};
    const cudaError_t err = launch(fn, dim3((unsigned)std::min<int64_t>(std::max<int64_t>(1, ceil_div(threads, 256)), 30LL * sm_count())), 256, args,
                                   static_cast<cudaStream_t>(stream));
    return err == cudaSuccess ? VQC_OK : cuda_error(err, "dropout launch");
}

}  // namespace
}  // namespace layers
}  // namespace vqc

using namespace vqc;

extern "C" {

vqc_status vqc_dropout_forward(vqc_real dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
                               int64_t residual_stride, double p, uint64_t seed, uint64_t offset, const uint64_t* state, void* y,
                               void* stream) {
    try {
        return layers::dropout("vqc_dropout_forward", dtype, rows, cols, x, x_stride, residual, residual_stride, p, seed, offset, state, y, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_dropout_backward(vqc_real dtype, int64_t rows, int64_t cols, const void* grad_y, int64_t grad_y_stride, double p,
                                uint64_t seed, uint64_t offset, const uint64_t* state, void* grad_x, void* stream) {
    try {
        return layers::dropout("vqc_dropout_backward", dtype, rows, cols, grad_y, grad_y_stride, nullptr, 0, p, seed, offset, state, grad_x, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
