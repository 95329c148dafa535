// layers_product.cu -- matrix products on the FP32 units, for every type,
// layout, stride and size, and the join of products that were cut along the
// contraction.
//
// Operands become float in shared memory, sums are float FMAs in a fixed order.
#include <algorithm>

#include "layers_elem.cuh"
#include "layers_tc.h"

namespace vqc {
namespace layers {

vqc_status cuda_error(cudaError_t e, const char* what) {
    return set_error(VQC_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
        cudaGetLastError();
        return 152;
    }
    return sms;
}

namespace {

struct ProductArgs {
    Operand a[2], b[2];
    Finish f;
    int64_t k;
    float* part;     // [splits][2 or 1][m][n] sums of a cut contraction, or NULL
    int32_t form, splits;
    int64_t tiles_m, tiles_n;
};

// A BM x BN tile of outputs per CTA of 256 threads, BK contracted elements at a
// time.  Each thread holds TM x TN sums: columns tx * TN/2 + [0, TN/2) of both
// halves of the tile.  In GATED form the first half of the tile's columns
// belongs to b0 and the second half to b1 (the same outputs), so that both
// factors of an output meet in one thread.
template <typename T, int BM, int BN, int TM, int TN>
__global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ ProductArgs A) {
    constexpr int BK = 16, NT = 256, TX = BN / TN;
    static_assert((BM / TM) * TX == NT && TN % 2 == 0, "tile");
    __shared__ float sa[BK][BM + 4], sb[BK][BN + 4];
    const int tid = threadIdx.x, tx = tid % TX, ty = tid / TX;
    const bool gated = A.form == GATED;
    const int64_t tile = blockIdx.x / A.tiles_n;
    const int64_t n0 = (blockIdx.x % A.tiles_n) * (gated ? BN / 2 : BN), m0 = tile % A.tiles_m * BM;
    const int split = (int)(tile / A.tiles_m), which = blockIdx.y;
    const int64_t m = A.f.m, n = A.f.n;
    const int64_t blocks = (A.k + BK - 1) / BK, terms = A.form == SUM ? 2 : 1;
    const int64_t kb0 = blocks * terms * split / A.splits, kb1 = blocks * terms * (split + 1) / A.splits;

    float acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = 0.f;

    for (int64_t kb = kb0; kb < kb1; ++kb) {
        const int term = kb >= blocks ? 1 : 0;
        const int64_t k0 = (kb - term * blocks) * BK;
        const Operand oa = A.a[which + term], ob = A.b[which + term];
        const T* pa = static_cast<const T*>(oa.p);
        for (int e = tid; e < BM * BK; e += NT) {
            const int i = oa.k_outer ? e % BM : e / BK, kk = oa.k_outer ? e / BM : e % BK;
            const int64_t r = m0 + i, c = k0 + kk;
            sa[kk][i] = r < m && c < A.k ? to_f(pa[oa.k_outer ? c * oa.ld + r : r * oa.ld + c]) : 0.f;
        }
        for (int e = tid; e < BN * BK; e += NT) {
            const int i = ob.k_outer ? e % BN : e / BK, kk = ob.k_outer ? e / BN : e % BK;
            const bool up = gated && i >= BN / 2;
            const T* pb = static_cast<const T*>(up ? A.b[1].p : ob.p);
            const int64_t ld = up ? A.b[1].ld : ob.ld, r = n0 + (up ? i - BN / 2 : i), c = k0 + kk;
            sb[kk][i] = r < n && c < A.k ? to_f(pb[ob.k_outer ? c * ld + r : r * ld + c]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < BK; ++kk) {
            float a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = sa[kk][ty * TM + i];
#pragma unroll
            for (int j = 0; j < TN / 2; ++j) {
                b[j] = sb[kk][tx * (TN / 2) + j];
                b[TN / 2 + j] = sb[kk][BN / 2 + tx * (TN / 2) + j];
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + ty * TM + i;
        if (row >= m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const bool second = j >= TN / 2;
            const int64_t c = tx * (TN / 2) + (second ? j - TN / 2 : j);
            const int64_t col = n0 + c + (second && !gated ? BN / 2 : 0);
            if (col >= n) continue;
            if (A.part) {
                const int64_t slot = gated ? 2 * split + second : (A.form == PAIR ? 2 * split + which : split);
                A.part[(slot * m + row) * n + col] = acc[i][j];
            } else if (!gated) {
                finish_one(A.f, which, row, col, acc[i][j], 0.f);
            } else if (!second) {
                finish_one(A.f, 0, row, col, acc[i][j], acc[i][TN / 2 + j]);
            }
        }
    }
}

// Sums of a cut contraction joined in the order of the cuts, then finished.
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Finish f, const float* part, int splits,
                                                   int form) {
    const int64_t size = f.m * f.n, step = (int64_t)gridDim.x * blockDim.x;
    const int which = blockIdx.y;
    const int64_t slots = form == GATED || form == PAIR ? 2 : 1;
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < size; e += step) {
        float v0 = 0.f, v1 = 0.f;
        for (int s = 0; s < splits; ++s) {
            v0 += part[(s * slots + which) * size + e];
            if (form == GATED) v1 += part[(s * slots + 1) * size + e];
        }
        finish_one(f, which, e / f.n, e % f.n, v0, v1);
    }
}

struct Tile {
    int bm, bn;
};

// Tiles by the number of outputs; few outputs over a long contraction are cut
// along it until the SMs have two CTAs each (cuts of at least 128 elements).
Tile pick_tile(const Product& p) {
    const int64_t cols = p.form == GATED ? 2 * p.n : p.n;
    if (cols <= 16) return {128, 16};
    return {64, 64};
}

int pick_splits(const Product& p, Tile t) {
    const int64_t tiles = ceil_div(p.m, t.bm) * ceil_div(p.n, p.form == GATED ? t.bn / 2 : t.bn) * (p.form == PAIR ? 2 : 1);
    const int64_t most = ceil_div(p.k * (p.form == SUM ? 2 : 1), 128);
    return (int)std::max<int64_t>(1, std::min<int64_t>({most, 2LL * sm_count() / std::max<int64_t>(tiles, 1), 64}));
}

template <typename T, int BM, int BN, int TM, int TN>
cudaError_t launch_product(ProductArgs a, cudaStream_t s) {
    a.tiles_m = ceil_div(a.f.m, BM);
    a.tiles_n = ceil_div(a.f.n, a.form == GATED ? BN / 2 : BN);
    const int64_t grid = a.tiles_m * a.tiles_n * a.splits;
    if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    void* args[] = {&a};
    return cudaLaunchKernel((const void*)product_kernel<T, BM, BN, TM, TN>, dim3((unsigned)grid, a.form == PAIR ? 2 : 1),
                            dim3(256), args, 0, s);
}

template <typename T> cudaError_t launch_tile(const ProductArgs& a, Tile t, cudaStream_t s) {
    if (t.bn == 16) return launch_product<T, 128, 16, 4, 2>(a, s);
    return launch_product<T, 64, 64, 4, 4>(a, s);
}

size_t part_bytes(const Product& p, int splits) {
    return splits > 1 ? align256((size_t)splits * (p.form == GATED || p.form == PAIR ? 2 : 1) * p.m * p.n * 4) : 0;
}

}  // namespace

vqc_status join_run(const Product& p, const float* part, int splits, cudaStream_t s) {
    Finish f = p.f;
    int form = p.form;
    const int64_t blocks = std::min<int64_t>(ceil_div(p.m * p.n, 256), 8LL * sm_count());
    void* args[] = {&f, &part, &splits, &form};
    const cudaError_t e = cudaLaunchKernel((const void*)join_kernel, dim3((unsigned)blocks, form == PAIR ? 2 : 1),
                                           dim3(256), args, 0, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "join launch");
}

size_t product_workspace(const Product& p, bool aligned) {
    if (p.m == 0 || p.k == 0) return 0;
    if (rows_takes(p)) return 0;
    if (tc_takes(p)) return tc_workspace(p, aligned);
    return part_bytes(p, pick_splits(p, pick_tile(p)));
}

vqc_status product_run(const Product& p, void* ws, size_t ws_bytes, cudaStream_t s) {
    if (p.m == 0 || p.n == 0) return VQC_OK;
    if (rows_takes(p)) return rows_run(p, s);
    if (tc_takes(p)) return tc_run(p, ws, ws_bytes, s);
    const Tile t = pick_tile(p);
    ProductArgs a{};
    for (int i = 0; i < 2; ++i) { a.a[i] = p.a[i]; a.b[i] = p.b[i]; }
    if (p.form == GATED) a.a[1] = p.a[0];
    a.f = p.f;
    a.k = p.k;
    a.form = p.form;
    a.splits = p.k == 0 ? 1 : pick_splits(p, t);
    const size_t need = part_bytes(p, a.splits);
    if (need > ws_bytes || (need && !ws)) return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
    a.part = need ? static_cast<float*>(ws) : nullptr;
    const cudaError_t e = p.f.dtype == VQC_F32    ? launch_tile<float>(a, t, s)
                          : p.f.dtype == VQC_BF16 ? launch_tile<__nv_bfloat16>(a, t, s)
                                                  : launch_tile<__half>(a, t, s);
    if (e != cudaSuccess) return cuda_error(e, "product launch");
    return need ? join_run(p, a.part, a.splits, s) : VQC_OK;
}

// ---------------------------------------------------------------- dz and column sums

namespace {

// One pass over grad_y and the saved pre-activations, bound by their bytes.  A CTA
// takes 256 columns x `per` rows: a thread owns 8 columns (neighbours where
// rows lie on 16-byte boundaries, else 32 apart) of every eighth row and keeps
// their sums in registers; these are joined over the CTA in shared memory
// and over the CTAs by sum_kernel, both in a fixed order.
constexpr int kGradCols = 256;

// 8 elements as they lie in memory, and as floats
struct Raw8 {
    uint32_t w[8];
};
template <bool VEC> __device__ __forceinline__ void load8(const void* p, int dtype, int64_t row, int64_t c, int64_t n, Raw8& v) {
    if constexpr (VEC) {
        if (dtype == VQC_F32) {
            const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + row + c);
            const uint4 a = __ldcs(q), b = __ldcs(q + 1);
            v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w;
            v.w[4] = b.x; v.w[5] = b.y; v.w[6] = b.z; v.w[7] = b.w;
        } else {
            const uint4 a = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + row + c));
            v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.w[i] = c + 32 * i < n ? __float_as_uint(load_as(p, dtype, row + c + 32 * i)) : 0u;
    }
}
template <bool VEC> __device__ __forceinline__ void floats8(const Raw8& r, int dtype, float (&v)[8]) {
    if (VEC && dtype != VQC_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = dtype == VQC_BF16 ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.w[i]))
                                               : __half22float2(*reinterpret_cast<const __half2*>(&r.w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void store8(void* p, int64_t row, int64_t c, int64_t n, const float (&v)[8]) {
    T o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = from_f<T>(v[i]);
    T* q = static_cast<T*>(p) + row + c;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(q)[i] = reinterpret_cast<const uint4*>(o)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + 32 * i < n) q[32 * i] = o[i];
    }
}

// The loads of UR rows are issued before the first of them is used.
template <typename T, bool VEC, int ACT, bool GATE>
__device__ __forceinline__ void act_grad_rows(const ActGrad& A, int64_t r0, int64_t r1, int64_t c, float (&s0)[8], float (&s1)[8]) {
    constexpr int UR = GATE ? 1 : 2;
    for (int64_t r = r0; r < r1; r += 8 * UR) {
        Raw8 rg[UR], rz[UR], ru[UR];
#pragma unroll
        for (int k = 0; k < UR; ++k) {
            const int64_t q = r + 8 * k;
            if (q >= r1) break;
            load8<VEC>(A.gy, A.gy_dtype, q * A.ld_gy, c, A.n, rg[k]);
            if (ACT != VQC_ACT_NONE || GATE) load8<VEC>(A.z[0], VQC_F32, q * A.n, c, A.n, rz[k]);
            if (GATE) load8<VEC>(A.z[1], VQC_F32, q * A.n, c, A.n, ru[k]);
        }
#pragma unroll
        for (int k = 0; k < UR; ++k) {
            const int64_t q = r + 8 * k;
            if (q >= r1) break;
            float gy[8], z[8], u[8], d[8];
            floats8<VEC>(rg[k], A.gy_dtype, gy);
            if (ACT != VQC_ACT_NONE || GATE) floats8<VEC>(rz[k], VQC_F32, z);
            if (GATE) floats8<VEC>(ru[k], VQC_F32, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (GATE) {
                    const float2 v = act_both(ACT, z[i]);
                    d[i] = gy[i] * u[i] * v.y;
                    u[i] = gy[i] * v.x;
                    s1[i] += u[i];
                } else {
                    d[i] = ACT == VQC_ACT_NONE ? gy[i] : gy[i] * act_both(ACT, z[i]).y;
                }
                s0[i] += d[i];
            }
            if (A.dz[0]) store8<T, VEC>(A.dz[0], q * A.ld_dz, c, A.n, d);
            if (GATE && A.dz[0]) store8<T, VEC>(A.dz[1], q * A.ld_dz, c, A.n, u);
        }
    }
}
template <typename T, bool VEC, bool GATE>
__device__ __forceinline__ void act_grad_as(const ActGrad& A, int64_t r0, int64_t r1, int64_t c, float (&s0)[8], float (&s1)[8]) {
    switch (A.act) {
        case VQC_ACT_RELU: return act_grad_rows<T, VEC, VQC_ACT_RELU, GATE>(A, r0, r1, c, s0, s1);
        case VQC_ACT_GELU: return act_grad_rows<T, VEC, VQC_ACT_GELU, GATE>(A, r0, r1, c, s0, s1);
        case VQC_ACT_SILU: return act_grad_rows<T, VEC, VQC_ACT_SILU, GATE>(A, r0, r1, c, s0, s1);
        case VQC_ACT_TANH: return act_grad_rows<T, VEC, VQC_ACT_TANH, GATE>(A, r0, r1, c, s0, s1);
        case VQC_ACT_SIGMOID: return act_grad_rows<T, VEC, VQC_ACT_SIGMOID, GATE>(A, r0, r1, c, s0, s1);
        default: return act_grad_rows<T, VEC, VQC_ACT_NONE, GATE>(A, r0, r1, c, s0, s1);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 3) act_grad_kernel(const __grid_constant__ ActGrad A, float* part, int64_t per) {
    __shared__ float sums[8][kGradCols];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t across = (A.n + kGradCols - 1) / kGradCols, block = blockIdx.x / across, blocks = gridDim.x / across;
    const int64_t c0 = blockIdx.x % across * kGradCols, c = c0 + (VEC ? 8 * lane : lane);
    float s0[8] = {}, s1[8] = {};
    if (c < A.n) {
        const int64_t r0 = block * per + warp, r1 = min(A.rows, (block + 1) * per);
        if (A.gated) act_grad_as<T, VEC, true>(A, r0, r1, c, s0, s1);
        else act_grad_as<T, VEC, false>(A, r0, r1, c, s0, s1);
    }
    if (!part) return;
    for (int w = 0; w < (A.gated ? 2 : 1); ++w) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[warp][VEC ? 8 * lane + i : lane + 32 * i] = w ? s1[i] : s0[i];
        __syncthreads();
        if (c0 + threadIdx.x < A.n) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += sums[i][threadIdx.x];
            part[(w * blocks + block) * A.n + c0 + threadIdx.x] = v;
        }
    }
}

// 32 columns per CTA: warp w adds the rows w, w + 32, ..., then the 32 sums are added.
__global__ void __launch_bounds__(1024) sum_kernel(const float* part, int64_t count, int64_t n, void* out0, void* out1,
                                                   int dtype) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    void* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    part += (int64_t)blockIdx.y * count * n;
    float v = 0.f;
    if (c < n)
#pragma unroll 4
        for (int64_t i = warp; i < count; i += 32) v += part[i * n + c];
    sums[warp][lane] = v;
    __syncthreads();
    // transposed, so that a warp joins the sums of one column
    v = sums[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < n) store_as(out, dtype, (int64_t)blockIdx.x * 32 + warp, v);
}

// Rows of a CTA: enough CTAs for four per SM, at least 16 rows, at most 256
int64_t grad_rows(int64_t rows, int64_t n) {
    const int64_t want = ceil_div(rows * ceil_div(n, kGradCols), 4LL * sm_count());
    return std::min<int64_t>(256, std::max<int64_t>(16, (want + 7) / 8 * 8));
}

}  // namespace

vqc_status sum_run(const float* part, int64_t count, int64_t n, void* out0, void* out1, int dtype, cudaStream_t s) {
    void* args[] = {&part, &count, &n, &out0, &out1, &dtype};
    const cudaError_t e = cudaLaunchKernel((const void*)sum_kernel, dim3((unsigned)ceil_div(n, 32), out1 ? 2 : 1),
                                           dim3(1024), args, 0, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "sum launch");
}

size_t act_grad_workspace(int64_t rows, int64_t n, bool gated) {
    return align256((size_t)std::max<int64_t>(1, ceil_div(rows, grad_rows(rows, n))) * n * (gated ? 2 : 1) * 4);
}

vqc_status act_grad_run(const ActGrad& a0, void* ws, size_t ws_bytes, cudaStream_t s) {
    ActGrad a = a0;
    const bool sums = a.sum[0] != nullptr;
    float* part = sums ? static_cast<float*>(ws) : nullptr;
    if (sums && (!ws || ws_bytes < act_grad_workspace(a.rows, a.n, a.gated)))
        return set_error(VQC_ERR_WORKSPACE, "column sums: workspace too small");
    int64_t per = grad_rows(a.rows, a.n);
    const int64_t blocks = ceil_div(a.rows, per), grid = blocks * ceil_div(a.n, kGradCols);
    if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "too many rows times columns");
    if (grid > 0) {
        // whole packs of 8 elements on 16-byte boundaries (z is dense, dz the library's own)
        const bool vec = a.n % 8 == 0 && a.ld_gy % 8 == 0 && aligned_to(a.gy, 16) && aligned_to(a.z[0], 16) && aligned_to(a.z[1], 16);
        void* args[] = {&a, &part, &per};
        const void* fn = a.dtype == VQC_F32 ? (vec ? (const void*)act_grad_kernel<float, true> : (const void*)act_grad_kernel<float, false>)
                         : a.dtype == VQC_BF16 ? (vec ? (const void*)act_grad_kernel<__nv_bfloat16, true> : (const void*)act_grad_kernel<__nv_bfloat16, false>)
                                               : (vec ? (const void*)act_grad_kernel<__half, true> : (const void*)act_grad_kernel<__half, false>);
        const cudaError_t e = cudaLaunchKernel(fn, dim3((unsigned)grid), dim3(256), args, 0, s);
        if (e != cudaSuccess) return cuda_error(e, "activation gradient launch");
    }
    return sums ? sum_run(part, blocks, a.n, a.sum[0], a.gated ? a.sum[1] : nullptr, a.dtype, s) : VQC_OK;
}

}  // namespace layers
}  // namespace vqc
