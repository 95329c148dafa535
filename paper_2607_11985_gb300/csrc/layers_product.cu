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
    if (tc_takes(p)) return tc_workspace(p, aligned);
    return part_bytes(p, pick_splits(p, pick_tile(p)));
}

vqc_status product_run(const Product& p, void* ws, size_t ws_bytes, cudaStream_t s) {
    if (p.m == 0 || p.n == 0) return VQC_OK;
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

constexpr int kGradRows = 64;   // rows of one CTA

// A CTA takes 128 columns x kGradRows rows: warp w the rows w, w + 8, ..., lane l
// the columns l + 32 i.  Column sums are joined over the warps in shared memory
// and over the CTAs by sum_kernel, both in a fixed order.
template <typename T>
__global__ void __launch_bounds__(256) act_grad_kernel(const __grid_constant__ ActGrad A, float* part) {
    __shared__ float sums[2][8][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t across = (A.n + 127) / 128, block = blockIdx.x / across, blocks = gridDim.x / across;
    const int64_t c0 = blockIdx.x % across * 128, r0 = block * kGradRows;
    float s0[4] = {}, s1[4] = {};
    for (int i = warp; i < kGradRows; i += 8) {
        const int64_t r = r0 + i;
        if (r >= A.rows) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = c0 + lane + 32 * j;
            if (c >= A.n) continue;
            const float gy = load_as(A.gy, A.gy_dtype, r * A.ld_gy + c);
            float d0, d1 = 0.f;
            if (A.gated) {
                const float2 v = act_both(A.act, A.z[0][r * A.n + c]);
                d0 = gy * A.z[1][r * A.n + c] * v.y;
                d1 = gy * v.x;
                if (A.dz[1]) static_cast<T*>(A.dz[1])[r * A.ld_dz + c] = from_f<T>(d1);
            } else {
                d0 = A.act == VQC_ACT_NONE ? gy : gy * act_both(A.act, A.z[0][r * A.n + c]).y;
            }
            if (A.dz[0]) static_cast<T*>(A.dz[0])[r * A.ld_dz + c] = from_f<T>(d0);
            s0[j] += d0;
            s1[j] += d1;
        }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sums[0][warp][lane + 32 * j] = s0[j];
        sums[1][warp][lane + 32 * j] = s1[j];
    }
    __syncthreads();
    const int c = threadIdx.x & 127, w = threadIdx.x >> 7;
    if (c0 + c < A.n && (w == 0 || A.gated)) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[w][i][c];
        part[(w * blocks + block) * A.n + c0 + c] = v;
    }
}

// out[c] = sum over i of part[i][c], in the order of i: 32 columns per CTA, warp w
// adds the rows w, w + 8, ..., then the eight sums.
__global__ void __launch_bounds__(256) sum_kernel(const float* part, int64_t count, int64_t n, void* out0, void* out1,
                                                  int dtype) {
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    part += (int64_t)blockIdx.y * count * n;
    float v = 0.f;
    if (c < n)
        for (int64_t i = warp; i < count; i += 8) v += part[i * n + c];
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < n) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[i][lane];
        store_as(blockIdx.y ? out1 : out0, dtype, c, v);
    }
}

}  // namespace

vqc_status sum_run(const float* part, int64_t count, int64_t n, void* out0, void* out1, int dtype, cudaStream_t s) {
    void* args[] = {&part, &count, &n, &out0, &out1, &dtype};
    const cudaError_t e = cudaLaunchKernel((const void*)sum_kernel, dim3((unsigned)ceil_div(n, 32), out1 ? 2 : 1),
                                           dim3(256), args, 0, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "sum launch");
}

size_t act_grad_workspace(int64_t rows, int64_t n, bool gated) {
    return align256((size_t)std::max<int64_t>(1, ceil_div(rows, kGradRows)) * n * (gated ? 2 : 1) * 4);
}

vqc_status act_grad_run(const ActGrad& a0, void* ws, size_t ws_bytes, cudaStream_t s) {
    ActGrad a = a0;
    const bool sums = a.sum[0] != nullptr;
    float* part = sums ? static_cast<float*>(ws) : nullptr;
    if (sums && (!ws || ws_bytes < act_grad_workspace(a.rows, a.n, a.gated)))
        return set_error(VQC_ERR_WORKSPACE, "column sums: workspace too small");
    const int64_t blocks = ceil_div(a.rows, kGradRows);
    const int64_t grid = blocks * ceil_div(a.n, 128);
    if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "too many rows times columns");
    if (grid > 0) {
        void* args[] = {&a, &part};
        const void* fn = a.dtype == VQC_F32    ? (const void*)act_grad_kernel<float>
                         : a.dtype == VQC_BF16 ? (const void*)act_grad_kernel<__nv_bfloat16>
                                               : (const void*)act_grad_kernel<__half>;
        const cudaError_t e = cudaLaunchKernel(fn, dim3((unsigned)grid), dim3(256), args, 0, s);
        if (e != cudaSuccess) return cuda_error(e, "activation gradient launch");
    }
    return sums ? sum_run(part, blocks, a.n, a.sum[0], a.gated ? a.sum[1] : nullptr, a.dtype, s) : VQC_OK;
}

}  // namespace layers
}  // namespace vqc
