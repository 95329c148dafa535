// layers_product.cu -- matrix products on the FP32 units, the join of products that
// were cut along the contraction, and the pass over dz of a backward.
//
// 16-bit operands go to the tensor cores, products with few rows to
// layers_rows.cu; what is left here are float products of moderate size, for
// every layout, stride and size, with sums in a fixed order.
#include <algorithm>
#include <atomic>
#include <mutex>
#include <set>
#include <type_traits>
#include <utility>

#include "layers_elem.cuh"
#include "layers_tc.h"

namespace vqc {
namespace layers {

vqc_status cuda_error(cudaError_t e, const char* what) {
    return set_error(VQC_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

cudaError_t launch(const void* fn, dim3 grid, int threads, void** args, cudaStream_t s, size_t shared, int cluster) {
    if (shared > 32 * 1024) {     // with a kernel's static shared memory, possibly above the default limit
        static std::mutex mu;
        static std::set<std::pair<const void*, int>> raised;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        std::lock_guard<std::mutex> lk(mu);
        if (!raised.count({fn, dev})) {      // one size per kernel: the launches of a kernel ask for no other
            e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
            if (e != cudaSuccess) return e;
            raised.insert({fn, dev});
        }
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (programmatic_launches()) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = cluster;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cudaLaunchKernelExC(&cfg, fn, args);
}

int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) == cudaSuccess) {
        if (dev < 64 && (sms = known[dev].load())) return sms;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0) {
            if (dev < 64) known[dev].store(sms);
            return sms;
        }
    }
    cudaGetLastError();
    return 152;
}

namespace {

struct ProductArgs {
    Operand a[2], b[2];
    Finish f;
    int64_t k;
    float* part;     // sums of a cut contraction, or NULL
    int32_t form, splits, vec_a, vec_b;
    int64_t tiles_m, tiles_n, ctas;
};
// Up to two products of one launch, the CTAs of the first before those of the second.
struct ProductPair {
    ProductArgs p[2];
};

constexpr int BK = 16, NT = 256;

// The elements of a tile of W outer rows x BK contracted that one thread moves:
// groups of 4 neighbours in memory, one 16-byte load each where `vec` allows.
template <int W> struct Slice {
    static constexpr int kGroups = (W * BK / 4 + NT - 1) / NT;
    float v[kGroups][4];

    __device__ __forceinline__ void load(const Operand& o, const float* second, int64_t ld, bool vec, int64_t i0, int64_t outer, int64_t k0, int64_t k,
                                         int split_at) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int e = threadIdx.x + g * NT;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[g][j] = 0.f;
            if (W * BK / 4 < NT && e >= W * BK / 4) continue;
            int i = o.k_outer ? e % (W / 4) * 4 : e / (BK / 4);
            const int kk = o.k_outer ? e / (W / 4) : e % (BK / 4) * 4;
            const float* p = static_cast<const float*>(o.p);
            if (second && i >= split_at) {
                p = second;
                i -= split_at;
            }
            const int64_t r = i0 + i, c = k0 + kk;
            const int64_t at = o.k_outer ? c * ld + r : r * ld + c;
            const int64_t inner = o.k_outer ? outer - r : k - c;     // elements left in this direction
            if (o.k_outer ? c >= k : r >= outer) continue;
            if (vec && inner >= 4) {
                const float4 q = *reinterpret_cast<const float4*>(p + at);
                v[g][0] = q.x; v[g][1] = q.y; v[g][2] = q.z; v[g][3] = q.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < inner) v[g][j] = p[at + j];
            }
        }
    }
    __device__ __forceinline__ void store(float (*s)[W + 4], bool k_outer) const {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int e = threadIdx.x + g * NT;
            if (W * BK / 4 < NT && e >= W * BK / 4) continue;
            if (k_outer) {
                *reinterpret_cast<float4*>(&s[e / (W / 4)][e % (W / 4) * 4]) = make_float4(v[g][0], v[g][1], v[g][2], v[g][3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) s[e % (BK / 4) * 4 + j][e / (BK / 4)] = v[g][j];
            }
        }
    }
};

// y = finish(A B^T) in float FMAs: a BM x BN tile of outputs per CTA of 256 threads, 16 contracted
// elements at a time, the next ones in flight meanwhile.  Bound by latency at the sizes
// that come here: 512 x 16 to 1024 11 us, 512 x 512 x 512 18.7 us (14 TFLOP/s), a chain of
// loads, a barrier and 16 steps per slice at two CTAs per SM.  Each thread holds TM x TN sums (packed pairs along n): columns
// tx * TN/2 + [0, TN/2) of both halves of the tile.  In GATED form the first
// half of the tile's columns belongs to b0 and the second half to b1 (the same
// outputs), so that both factors of an output meet in one thread.
template <int BM, int BN, int TM, int TN>
__global__ void __launch_bounds__(NT) product_kernel(const __grid_constant__ ProductPair P) {
    stream_order();
    constexpr int TX = BN / TN, TH = TN / 2;
    static_assert((BM / TM) * TX == NT && TN % 2 == 0, "tile");
    __shared__ __align__(16) float sa[2][BK][BM + 4], sb[2][BK][BN + 4];
    const int tid = threadIdx.x, tx = tid % TX, ty = tid / TX;
    int64_t block = blockIdx.x;
    const int which_product = block >= P.p[0].ctas ? 1 : 0;
    const ProductArgs& A = P.p[which_product];
    if (which_product) block -= P.p[0].ctas;
    const bool gated = A.form == GATED;
    int64_t tile = block / A.tiles_n;
    const int64_t n0 = block % A.tiles_n * (gated ? BN / 2 : BN), m0 = tile % A.tiles_m * BM;
    tile /= A.tiles_m;
    const int split = (int)(tile % A.splits), which = (int)(tile / A.splits);
    const int64_t m = A.f.m, n = A.f.n;
    const int64_t blocks = (A.k + BK - 1) / BK, terms = A.form == SUM ? 2 : 1;
    const int64_t kb0 = blocks * terms * split / A.splits, kb1 = blocks * terms * (split + 1) / A.splits;

    float acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = 0.f;

    Slice<BM> na;
    Slice<BN> nb;
    auto load = [&](int64_t kb) {
        const int term = kb >= blocks ? 1 : 0;
        const int64_t k0 = (kb - term * blocks) * BK;
        na.load(A.a[which + term], nullptr, A.a[which + term].ld, A.vec_a, m0, m, k0, A.k, BM);
        nb.load(A.b[which + term], gated ? static_cast<const float*>(A.b[1].p) : nullptr, A.b[which + term].ld, A.vec_b, n0, n, k0, A.k, BN / 2);
    };
    if (kb0 < kb1) load(kb0);
    int buf = 0;
    for (int64_t kb = kb0; kb < kb1; ++kb, buf ^= 1) {
        na.store(sa[buf], A.a[0].k_outer);
        nb.store(sb[buf], A.b[0].k_outer);
        __syncthreads();       // the other buffer was read before the barrier of the step before
        if (kb + 1 < kb1) load(kb + 1);
#pragma unroll
        for (int kk = 0; kk < BK; ++kk) {
            float a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = sa[buf][kk][ty * TM + i];
#pragma unroll
            for (int j = 0; j < TH; ++j) {
                b[j] = sb[buf][kk][tx * TH + j];
                b[TH + j] = sb[buf][kk][BN / 2 + tx * TH + j];
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; j += 2) {
                    const float2 r = fma2(make_float2(a[i], a[i]), make_float2(b[j], b[j + 1]), make_float2(acc[i][j], acc[i][j + 1]));
                    acc[i][j] = r.x;
                    acc[i][j + 1] = r.y;
                }
        }
    }
    let_next();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + ty * TM + i;
        if (row >= m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const bool second = j >= TH;
            const int64_t c = tx * TH + (second ? j - TH : j);
            const int64_t col = n0 + c + (second && !gated ? BN / 2 : 0);
            if (col >= n) continue;
            if (A.part) {
                const int64_t slot = gated ? 2 * split + second : (A.form == PAIR ? 2 * split + which : split);
                A.part[(slot * m + row) * n + col] = acc[i][j];
            } else if (!gated) {
                finish_one(A.f, which, row, col, acc[i][j], 0.f);
            } else if (!second) {
                finish_one(A.f, 0, row, col, acc[i][j], acc[i][TH + j]);
            }
        }
    }
}

// Sums of cut contractions joined in the order of the cuts, then finished (bound by the launch: its
// operands lie in the L2): job
// blockIdx.y / 2, its product blockIdx.y % 2 (PAIR).  Four neighbouring outputs per
// thread where a row holds a multiple of four.
template <int W> __device__ __forceinline__ void join_at(const Join& j, int which, int64_t size, int64_t stride, int64_t e) {
    const float* p = j.part + which * size + e;
    float v0[W], v1[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v0[i] = v1[i] = 0.f;
    auto add = [&](const float* q, float (&v)[W]) {
        if constexpr (W == 4) {
            const float4 f = *reinterpret_cast<const float4*>(q);
            v[0] += f.x; v[1] += f.y; v[2] += f.z; v[3] += f.w;
        } else {
            v[0] += *q;
        }
    };
    if (j.form == GATED) {
#pragma unroll 4
        for (int s = 0; s < j.splits; ++s) {
            add(p + s * stride, v0);
            add(p + s * stride + size, v1);
        }
    } else {
#pragma unroll 8
        for (int s = 0; s < j.splits; ++s) add(p + s * stride, v0);
    }
    // most outputs count less than 2^32 elements: a short division
    const int64_t row = size >> 32 ? e / j.f.n : (int64_t)((uint32_t)e / (uint32_t)j.f.n), col = e - row * j.f.n;
    finish_some<W>(j.f, which, row, col, v0, v1);
}
// One row of many cuts (column sums): a warp's lanes take 32 columns, warp w the cuts w,
// w + 8, ..., then the eight sums are added.
__device__ __forceinline__ void join_row(const Join& j, int which, int64_t stride) {
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = j.f.n;
    for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < n; c0 += (int64_t)gridDim.x * 32) {
        float v = 0.f;
        if (c0 + lane < n) {
            const float* p = j.part + which * n + c0 + lane;
#pragma unroll 8
            for (int s = warp; s < j.splits; s += 8) v += p[s * stride];
        }
        sums[warp][lane] = v;
        __syncthreads();
        if (warp == 0 && c0 + lane < n) {
            v = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += sums[i][lane];
            finish_one(j.f, which, 0, c0 + lane, v, 0.f);
        }
        __syncthreads();
    }
}
__global__ void __launch_bounds__(256, 2) join_kernel(const __grid_constant__ Joins J) {
    stream_order();
    const Join& j = J.j[blockIdx.y >> 1];
    const int which = blockIdx.y & 1;
    if (which && j.form != PAIR) return;
    const int64_t size = j.f.m * j.f.n, step = (int64_t)gridDim.x * blockDim.x, at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t stride = size * (j.form == GATED || j.form == PAIR ? 2 : 1);
    if (j.f.m == 1 && j.form != GATED && j.splits >= 8) {
        join_row(j, which, stride);
    } else if (j.f.n % 4 == 0) {
        for (int64_t e = 4 * at; e < size; e += 4 * step) join_at<4>(j, which, size, stride, e);
    } else {
        for (int64_t e = at; e < size; e += step) join_at<1>(j, which, size, stride, e);
    }
}

struct Tile {
    int bm, bn;
};

// Tiles by the number of outputs' columns; few outputs over a long contraction are cut
// along it until the SMs have two CTAs each (cuts of at least 64 elements).
Tile pick_tile(const Product& p) {
    const int64_t cols = p.form == GATED ? 2 * p.n : p.n;
    if (cols <= 16) return {128, 16};
    return {64, 64};
}

int pick_splits(const Product& p, Tile t) {
    if (p.k == 0) return 1;
    const int64_t tiles = ceil_div(p.m, t.bm) * ceil_div(p.n, p.form == GATED ? t.bn / 2 : t.bn) * (p.form == PAIR ? 2 : 1);
    const int64_t most = ceil_div(p.k * (p.form == SUM ? 2 : 1), 64);
    return (int)std::max<int64_t>(1, std::min<int64_t>({most, 2LL * sm_count() / std::max<int64_t>(tiles, 1), 64}));
}

size_t part_bytes(const Product& p, int splits) {
    return splits > 1 ? align256((size_t)splits * (p.form == GATED || p.form == PAIR ? 2 : 1) * p.m * p.n * 4) : 0;
}

// rows of float operands on 16-byte boundaries
bool packed(const Operand& o) { return o.ld % 4 == 0 && aligned_to(o.p, 16); }

vqc_status product_args(const Product& p, Tile t, void* ws, size_t ws_bytes, ProductArgs& a, Joins& joins) {
    for (int i = 0; i < 2; ++i) { a.a[i] = p.a[i]; a.b[i] = p.b[i]; }
    const int na = p.form == SUM || p.form == PAIR ? 2 : 1, nb = p.form == PLAIN ? 1 : 2;
    a.vec_a = packed(p.a[0]) && (na == 1 || packed(p.a[1]));
    a.vec_b = packed(p.b[0]) && (nb == 1 || packed(p.b[1]));
    a.f = p.f;
    a.k = p.k;
    a.form = p.form;
    a.splits = pick_splits(p, t);
    a.tiles_m = ceil_div(p.m, t.bm);
    a.tiles_n = ceil_div(p.n, p.form == GATED ? t.bn / 2 : t.bn);
    a.ctas = a.tiles_m * a.tiles_n * a.splits * (p.form == PAIR ? 2 : 1);
    const size_t need = part_bytes(p, a.splits);
    if (need > ws_bytes || (need && !ws)) return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
    a.part = need ? static_cast<float*>(ws) : nullptr;
    if (need) {
        Join& j = joins.j[joins.count++];
        j.f = p.f;
        j.part = a.part;
        j.splits = a.splits;
        j.form = p.form;
    }
    return VQC_OK;
}

}  // namespace

vqc_status join_run(const Joins& joins, cudaStream_t s) {
    if (!joins.count) return VQC_OK;
    int64_t most = 1;
    for (int i = 0; i < joins.count; ++i) most = std::max(most, joins.j[i].f.m * joins.j[i].f.n * (joins.j[i].f.m == 1 ? 8 : 1));
    void* args[] = {const_cast<Joins*>(&joins)};
    const cudaError_t e = launch((const void*)join_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(most, 256), 8LL * sm_count()), 2 * joins.count),
                                 256, args, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "join launch");
}

void products_workspace(const Product* p, int count, bool aligned, size_t* bytes) {
    Product tc[2];
    int index[2], have = 0;
    for (int i = 0; i < count; ++i) {
        bytes[i] = 0;
        if (p[i].m == 0 || rows_takes(p[i], aligned)) continue;
        if (tc_takes(p[i])) {
            tc[have] = p[i];
            index[have++] = i;
        } else {
            bytes[i] = part_bytes(p[i], pick_splits(p[i], pick_tile(p[i])));
        }
    }
    if (!have) return;
    size_t need[2];
    tc_workspace(tc, have, aligned, need);
    for (int i = 0; i < have; ++i) bytes[index[i]] = need[i];
}

vqc_status products_run(const Product* p, int count, void* const* ws, const size_t* bytes, Joins& joins, cudaStream_t s) {
    ProductPair pair[2]{};       // those of tiles 64 x 64, those of tiles 128 x 16
    int have[2] = {0, 0}, tcs = 0;
    Product tc[2];
    void* tc_ws[2];
    size_t tc_bytes[2];
    for (int i = 0; i < count; ++i) {
        if (p[i].m == 0 || p[i].n == 0) continue;
        vqc_status st = VQC_OK;
        const bool aligned = aligned_to(p[i].a[0].p, 16) && aligned_to(p[i].b[0].p, 16) && aligned_to(p[i].b[1].p, 16);
        if (rows_takes(p[i], aligned)) {
            st = rows_run(p[i], aligned, s);
        } else if (tc_takes(p[i])) {
            tc[tcs] = p[i];
            tc_ws[tcs] = ws[i];
            tc_bytes[tcs++] = bytes[i];
        } else {
            const Tile t = pick_tile(p[i]);
            const int kind = t.bn == 16;
            st = product_args(p[i], t, ws[i], bytes[i], pair[kind].p[have[kind]++], joins);
        }
        if (st != VQC_OK) return st;
    }
    if (tcs) {
        const vqc_status st = tc_run(tc, tcs, tc_ws, tc_bytes, joins, s);
        if (st != VQC_OK) return st;
    }
    for (int kind = 0; kind < 2; ++kind) {
        if (!have[kind]) continue;
        const int64_t grid = pair[kind].p[0].ctas + pair[kind].p[1].ctas;
        if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "product: too many tiles");
        void* args[] = {&pair[kind]};
        const void* fn = kind ? (const void*)product_kernel<128, 16, 4, 2> : (const void*)product_kernel<64, 64, 4, 4>;
        const cudaError_t e = launch(fn, dim3((unsigned)grid), NT, args, s);
        if (e != cudaSuccess) return cuda_error(e, "product launch");
    }
    return VQC_OK;
}

// ---------------------------------------------------------------- dz and column sums

namespace {

// One pass over grad_y and the saved pre-activations, bound by their bytes: 8192 x 5632
// bfloat16, a gate, column sums alone, 80 us (461 MB, 5.8 TB/s); copies ahead into
// shared memory took 104 and kept the products that follow off the SMs.  A CTA
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
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + (row + c) * (dtype == VQC_F32 ? 4 : 2));
        const uint4 a = __ldcs(q);
        v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w;
        if (dtype == VQC_F32) {
            const uint4 b = __ldcs(q + 1);
            v.w[4] = b.x; v.w[5] = b.y; v.w[6] = b.z; v.w[7] = b.w;
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

// v cut towards zero to a value of T, one step further towards zero, the smallest value of T
template <typename T> struct Cut;
template <> struct Cut<__nv_bfloat16> {
    static __device__ __forceinline__ float cut(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
    static __device__ __forceinline__ float before(float h) { return __uint_as_float(__float_as_uint(h) - 0x10000u); }
    static __device__ __forceinline__ float least() { return __uint_as_float(0x10000u); }
};
template <> struct Cut<__half> {
    static __device__ __forceinline__ float cut(float v) { return __half2float(__float2half_rz(v)); }
    static __device__ __forceinline__ float before(float h) { return __half2float(__ushort_as_half(__half_as_ushort(__float2half(h)) - 1)); }
    static __device__ __forceinline__ float least() { return 5.9604644775390625e-8f; }
};

// The first of the two parts that add up to a value; v becomes the second.  Both parts of a
// value other than zero have its sign and are not zero themselves, so that a factor that is
// infinite makes the one infinity of their products (zero or the other sign would make it
// NaN): the first is cut, and gives one unit to the second where nothing would be left.  What the
// smallest values of T add is a few of these.  Both parts of an infinity or NaN are that.
template <typename T> __device__ __forceinline__ float first_part(float& v) {
    if (v == 0.f || !(fabsf(to_f(from_f<T>(v))) <= 3.4028234e38f)) return v;
    float h = Cut<T>::cut(v);
    if (h == v) h = Cut<T>::before(h);
    if (h == 0.f) h = copysignf(Cut<T>::least(), v);
    v = copysignf(fmaxf(fabsf(v) - fabsf(h), Cut<T>::least()), v);
    return h;
}

// TWO: as two parts, the second A.second elements behind the first
template <typename T, bool VEC, bool TWO> __device__ __forceinline__ void store_dz(const ActGrad& A, int i, int64_t row, int64_t c, float (&v)[8]) {
    if constexpr (TWO) {
        float h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = first_part<T>(v[e]);
        store8<T, VEC>(A.dz[i], row, c, A.n, h);
        store8<T, VEC>(A.dz[i], row + A.second, c, A.n, v);
    } else {
        store8<T, VEC>(A.dz[i], row, c, A.n, v);
    }
}

// the largest of |v| that is finite, and `top`
__device__ __forceinline__ float top_of(float top, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (fabsf(v[i]) <= 3.4028234e38f) top = fmaxf(top, fabsf(v[i]));
    return top;
}

template <typename T, bool VEC, int ACT, bool GATE, bool TWO>
__device__ __forceinline__ void act_grad_rows(const ActGrad& A, int64_t r0, int64_t r1, int64_t c, float (&s0)[8], float (&s1)[8], float& top) {
    constexpr bool kScaled = std::is_same<T, __half>::value;
    const float scale = kScaled && A.scale && A.dz[0] ? A.scale[0] : 1.f;
    for (int64_t q = r0; q < r1; q += 8) {
        Raw8 rg, rz, ru;
        load8<VEC>(A.gy, A.gy_dtype, q * A.ld_gy, c, A.n, rg);
        if (ACT != VQC_ACT_NONE || GATE) load8<VEC>(A.z[0], VQC_F32, q * A.n, c, A.n, rz);
        if (GATE) load8<VEC>(A.z[1], VQC_F32, q * A.n, c, A.n, ru);
        float gy[8], z[8], u[8], d[8];
        floats8<VEC>(rg, A.gy_dtype, gy);
        if (ACT != VQC_ACT_NONE || GATE) floats8<VEC>(rz, VQC_F32, z);
        if (GATE) floats8<VEC>(ru, VQC_F32, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (GATE) {
                const float2 v = act_both<sizeof(T) == 4>(ACT, z[i]);
                // rounded products (not fused into the sums), whether or not dz is stored
                d[i] = __fmul_rn(__fmul_rn(gy[i], u[i]), v.y);
                u[i] = __fmul_rn(gy[i], v.x);
                s1[i] += u[i];
            } else {
                d[i] = ACT == VQC_ACT_NONE ? gy[i] : __fmul_rn(gy[i], act_both<sizeof(T) == 4>(ACT, z[i]).y);
            }
            s0[i] += d[i];
        }
        if constexpr (kScaled) {
            if (A.dz[0]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    d[i] *= scale;
                    if (GATE) u[i] *= scale;
                }
            } else if (A.scale) {
                top = top_of(top, d);
                if (GATE) top = top_of(top, u);
            }
        }
        if (A.dz[0]) store_dz<T, VEC, TWO>(A, 0, q * A.ld_dz, c, d);
        if (GATE && A.dz[0]) store_dz<T, VEC, TWO>(A, 1, q * A.ld_dz, c, u);
    }
}
template <typename T, bool VEC, bool GATE, bool TWO>
__device__ __forceinline__ void act_grad_as(const ActGrad& A, int64_t r0, int64_t r1, int64_t c, float (&s0)[8], float (&s1)[8], float& top) {
    switch (A.act) {
        case VQC_ACT_RELU: return act_grad_rows<T, VEC, VQC_ACT_RELU, GATE, TWO>(A, r0, r1, c, s0, s1, top);
        case VQC_ACT_GELU: return act_grad_rows<T, VEC, VQC_ACT_GELU, GATE, TWO>(A, r0, r1, c, s0, s1, top);
        case VQC_ACT_SILU: return act_grad_rows<T, VEC, VQC_ACT_SILU, GATE, TWO>(A, r0, r1, c, s0, s1, top);
        case VQC_ACT_TANH: return act_grad_rows<T, VEC, VQC_ACT_TANH, GATE, TWO>(A, r0, r1, c, s0, s1, top);
        case VQC_ACT_SIGMOID: return act_grad_rows<T, VEC, VQC_ACT_SIGMOID, GATE, TWO>(A, r0, r1, c, s0, s1, top);
        default: return act_grad_rows<T, VEC, VQC_ACT_NONE, GATE, TWO>(A, r0, r1, c, s0, s1, top);
    }
}

// CTAs per SM: by the registers
constexpr int grad_ctas(bool gate) { return gate ? 3 : 4; }
template <typename T, bool VEC, bool GATE, bool TWO>
__global__ void __launch_bounds__(256, grad_ctas(GATE)) act_grad_kernel(const __grid_constant__ ActGrad A, float* part, float* tops, int64_t per) {
    __shared__ float sums[8][kGradCols];
    stream_order();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t across = (A.n + kGradCols - 1) / kGradCols, block = blockIdx.x / across;
    const int64_t c0 = blockIdx.x % across * kGradCols, c = c0 + (VEC ? 8 * lane : lane);
    float s0[8] = {}, s1[8] = {}, top = 0.f;
    if (c < A.n) {
        const int64_t r0 = block * per + warp, r1 = min(A.rows, (block + 1) * per);
        act_grad_as<T, VEC, GATE, TWO>(A, r0, r1, c, s0, s1, top);
    }
    let_next();
    if (std::is_same<T, __half>::value && tops) {       // the CTA's largest magnitude
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        if (lane == 0) sums[0][warp] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 8; ++i) top = fmaxf(top, sums[0][i]);
            tops[blockIdx.x] = top;
        }
    }
    if (!part) return;
    for (int w = 0; w < (GATE ? 2 : 1); ++w) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[warp][VEC ? 8 * lane + i : lane + 32 * i] = w ? s1[i] : s0[i];
        __syncthreads();
        if (c0 + threadIdx.x < A.n) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += sums[i][threadIdx.x];
            part[(block * (GATE ? 2 : 1) + w) * A.n + c0 + threadIdx.x] = v;
        }
    }
}

// The power of two that brings the largest of `count` magnitudes to [2^14, 2^15), and its inverse;
// at least 1 where `up`.
__global__ void __launch_bounds__(1024) scale_kernel(const float* tops, int64_t count, int up, float* scale) {
    __shared__ float warps[32];
    stream_order();
    float top = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += 1024) top = fmaxf(top, tops[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 32; ++i) top = fmaxf(top, warps[i]);
        int e = top > 0.f ? min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 126) : 0;      // -113 at least
        if (up) e = max(e, 0);
        scale[0] = __uint_as_float((uint32_t)(127 + e) << 23);
        scale[1] = __uint_as_float((uint32_t)(127 - e) << 23);
    }
}

// The norm's column sums over its CTAs: 32 columns per CTA, warp w adds the rows w, w + 32, ...,
// then the 32 sums are added.  304 rows of 2 x 4096: 7 us, bound by latency.
__global__ void __launch_bounds__(1024) sum_kernel(const float* part, int64_t count, int64_t n, int64_t ld, int64_t second,
                                                   void* out0, void* out1, int dtype) {
    __shared__ float sums[32][33];
    stream_order();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    void* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    part += blockIdx.y * second;
    float v = 0.f;
    if (c < n)
#pragma unroll 8
        for (int64_t i = warp; i < count; i += 32) v += part[i * ld + c];
    sums[warp][lane] = v;
    __syncthreads();
    // transposed, so that a warp joins the sums of one column
    v = sums[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < n) store_as(out, dtype, (int64_t)blockIdx.x * 32 + warp, v);
}

// Rows of a CTA: as many CTAs as fit at one time, 16 to 256 rows each
int64_t grad_rows(int64_t rows, int64_t n, bool gate) {
    const int64_t want = ceil_div(rows * ceil_div(n, kGradCols), (int64_t)grad_ctas(gate) * sm_count());
    return std::min<int64_t>(256, std::max<int64_t>(16, (want + 7) / 8 * 8));
}
template <bool VEC, bool GATE> const void* grad_kernel(int dtype, bool two) {
    if (dtype == VQC_F32) return (const void*)act_grad_kernel<float, VEC, GATE, false>;
    if (dtype == VQC_BF16)
        return two ? (const void*)act_grad_kernel<__nv_bfloat16, VEC, GATE, true> : (const void*)act_grad_kernel<__nv_bfloat16, VEC, GATE, false>;
    return two ? (const void*)act_grad_kernel<__half, VEC, GATE, true> : (const void*)act_grad_kernel<__half, VEC, GATE, false>;
}

}  // namespace

vqc_status sum_run(const float* part, int64_t count, int64_t n, int64_t ld, int64_t second, void* out0, void* out1, int dtype,
                   cudaStream_t s) {
    void* args[] = {&part, &count, &n, &ld, &second, &out0, &out1, &dtype};
    const cudaError_t e = launch((const void*)sum_kernel, dim3((unsigned)ceil_div(n, 32), out1 ? 2 : 1), 1024, args, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "sum launch");
}

namespace {
size_t grad_sums_bytes(int64_t rows, int64_t n, bool gated) {
    return align256((size_t)std::max<int64_t>(1, ceil_div(rows, grad_rows(rows, n, gated))) * n * (gated ? 2 : 1) * 4);
}
int64_t grad_grid(int64_t rows, int64_t n, bool gated) { return ceil_div(rows, grad_rows(rows, n, gated)) * ceil_div(n, kGradCols); }
}  // namespace

size_t act_grad_workspace(int64_t rows, int64_t n, bool gated, bool scaled) {
    return grad_sums_bytes(rows, n, gated) + (scaled ? align256((size_t)grad_grid(rows, n, gated) * 4) : 0);
}

vqc_status act_grad_run(const ActGrad& a0, void* ws, size_t ws_bytes, Joins& joins, cudaStream_t s) {
    ActGrad a = a0;
    const bool sums = a.sum[0] != nullptr;
    float* part = sums ? static_cast<float*>(ws) : nullptr;
    if ((sums || a.scale) && (!ws || ws_bytes < act_grad_workspace(a.rows, a.n, a.gated, a.scale)))
        return set_error(VQC_ERR_WORKSPACE, "column sums: workspace too small");
    int64_t per = grad_rows(a.rows, a.n, a.gated);
    const int64_t blocks = ceil_div(a.rows, per);
    int64_t grid = grad_grid(a.rows, a.n, a.gated);
    if (grid > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, "too many rows times columns");
    if (grid > 0) {
        // whole packs of 8 elements on 16-byte boundaries (z is dense, dz the library's own)
        const bool vec = a.n % 8 == 0 && a.ld_gy % 8 == 0 && aligned_to(a.gy, 16) && aligned_to(a.z[0], 16) && aligned_to(a.z[1], 16);
        float* tops = nullptr;
        void* args[] = {&a, &part, &tops, &per};
        auto kernel = [&](bool two) {
            return vec ? (a.gated ? grad_kernel<true, true>(a.dtype, two) : grad_kernel<true, false>(a.dtype, two))
                       : (a.gated ? grad_kernel<false, true>(a.dtype, two) : grad_kernel<false, false>(a.dtype, two));
        };
        if (a.scale) {
            // float16 holds 2^-24 to 65504 only, and dz is an operand, not a result: what is small in
            // it counts in sums over many rows, and what is large (from a float32 grad_y) may meet small weights.
            // A first pass finds its largest magnitude (and the column sums), a second writes it times a
            // power of two, which the products' ends undo exactly: 2^-38 of the largest is kept.
            // A float16 grad_y is scaled up only: there a dz beyond 65504 stays infinite, the overflow that
            // training in float16 looks for.
            tops = reinterpret_cast<float*>(static_cast<char*>(ws) + grad_sums_bytes(a.rows, a.n, a.gated));
            a.dz[0] = a.dz[1] = nullptr;
            cudaError_t e = launch(kernel(false), dim3((unsigned)grid), 256, args, s);
            if (e != cudaSuccess) return cuda_error(e, "activation gradient launch");
            int up = a.gy_dtype == VQC_F16;
            void* of[] = {&tops, &grid, &up, &a.scale};
            e = launch((const void*)scale_kernel, dim3(1), 1024, of, s);
            if (e != cudaSuccess) return cuda_error(e, "scale launch");
            a.dz[0] = a0.dz[0];
            a.dz[1] = a0.dz[1];
            part = nullptr;
            tops = nullptr;
        }
        const cudaError_t e = launch(kernel(a.dz[0] && a.second), dim3((unsigned)grid), 256, args, s);
        if (e != cudaSuccess) return cuda_error(e, "activation gradient launch");
    }
    if (!sums) return VQC_OK;
    Join& j = joins.j[joins.count++];
    j.f.m = 1;
    j.f.n = a.n;
    j.f.dtype = j.f.out_dtype = a.dtype;
    j.f.y[0] = a.sum[0];
    j.f.y[1] = a.gated ? a.sum[1] : nullptr;
    j.part = static_cast<float*>(ws);
    j.splits = (int)blocks;
    j.form = a.gated ? PAIR : PLAIN;
    return VQC_OK;
}

}  // namespace layers
}  // namespace vqc
