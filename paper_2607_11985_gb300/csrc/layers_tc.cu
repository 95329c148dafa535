// layers_tc.cu -- products on the tensor cores (tcgen05).
//
// Float operands are multiplied as well: each is the sum of three bf16 parts, and
// the six products of parts down to 2^-16 of the whole are one contraction of
// six times the depth (what is dropped is about 2^-24 of the magnitudes, as a float's
// own rounding).
//
// One persistent kernel for every form: y = finish(A B^T) with A [m, k] and B
// [n, k] stored along k or along their outer index (the backward's products
// contract over rows: no operand is ever transposed in memory).
//
// A CTA, or a pair of CTAs on two SMs (cta_group::2), computes a tile of
// 128 x BN (256 x BN) outputs.  Warp 0 moves 64-deep slices of both operands
// into a ring of stages with TMA (128-byte swizzle; rows and columns beyond the
// matrix arrive as zeros), warp 1 issues the products of a stage (four of depth
// 16) into one of two accumulators in tensor memory, warps 4..11 take the other
// accumulator out, finish it (bias, activation, gate, residual, rounding) and
// write it while the next tile is multiplied.  In a pair each CTA holds its own
// 128 rows of A and half of B's rows, and the tensor cores of both read both
// halves: per CTA 32 KB arrive for 256 x 256 x 64 products instead of 48 KB for
// 128 x 256 x 64, which one SM's share of the L2 could not deliver in time.
// In GATED form half of the tile's columns are rows of the one weight and half
// of the other, so that both factors of an output lie in one lane.
//
// Every wait is bounded; one that runs out sets the error word, the CTAs drain
// their copies and products, free their tensor memory and return.
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "layers_elem.cuh"
#include "layers_tc.h"

namespace vqc {
namespace layers {

namespace {

constexpr int BM = 128, BK = 64;
constexpr int kThreads = 384, kEpiWarps = 8;
constexpr int kStageA = BM * BK * 2;                 // 16 KB
constexpr int kStaging = kEpiWarps * 2 * 32 * 17 * 4;   // transposition of unaligned outputs
constexpr int kBarriers = 1024;
constexpr int kSmemLimit = 232448;
constexpr unsigned long long kWaitNs = 4000000000ull;   // bound of every wait

template <int CG, int BN> struct Shape {
    static constexpr int kStageB = BN / CG * BK * 2;
    static constexpr int kStage = kStageA + kStageB;
    static constexpr int kStages = (kSmemLimit - kStaging - kBarriers) / kStage < 8 ? (kSmemLimit - kStaging - kBarriers) / kStage : 8;
    static constexpr int kSmem = kStages * kStage + kStaging + kBarriers;
    static constexpr int kTmem = 2 * BN;             // two accumulators, a power of two >= 32
};

// Maps of the operands: [operand][part].
template <int kParts> struct TcArgs {
    CUtensorMap ma[2][kParts], mb[2][kParts];
    Finish f;
    Exact exact;                // of float operands
    float* part;                // sums of a cut contraction, or NULL
    unsigned* err;
    int form, splits, tiles_m, tiles_n, kblocks, a_mn, b_mn, vec, bf16;
    long long tiles;
};

// Products of parts of float operands, small ones first: parts of a and b, 2 bits each.
constexpr unsigned kPartsA = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10;
constexpr unsigned kPartsB = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t at_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;\n" : "=l"(t));
    return t;
}
__device__ __forceinline__ void mbar_init(uint32_t mbar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(mbar), "r"(count) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t mbar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}\n"
        : "=r"(done)
        : "r"(mbar), "r"(parity)
        : "memory");
    return done != 0;
}

// Bounded wait for a phase; false when it ran out or another role gave up.
__device__ __noinline__ bool mbar_wait_slow(uint32_t mbar, uint32_t parity, const volatile int* gave_up) {
    const unsigned long long end = now_ns() + kWaitNs;
    for (unsigned i = 0;; ++i) {
        if (mbar_try(mbar, parity)) return true;
        if ((i & 63) == 63 && ((gave_up && *gave_up) || now_ns() > end)) return false;
    }
}
__device__ __forceinline__ bool mbar_wait(uint32_t mbar, uint32_t parity, const volatile int* gave_up) {
    if (mbar_try(mbar, parity)) return true;
    return mbar_wait_slow(mbar, parity, gave_up);
}

__device__ __forceinline__ void tma_prefetch(const CUtensorMap* m) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}
// One box at (x, y) into this CTA's shared memory; `mbar` may be the pair's first CTA's.
template <int CG> __device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t mbar) {
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, "
            "%3}], [%4];\n" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(mbar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n" ::"r"(
                dst),
            "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(mbar)
            : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle: start, leading byte offset
// (between chunks of 64 outer elements; unused along k), stride byte offset
// (between groups of 8 rows of 128 bytes), version 1.
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo) {
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

template <int CG> __device__ __forceinline__ void mma(uint32_t tmem, uint64_t a, uint64_t b, uint32_t idesc, int accumulate) {
    if (CG == 2)
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// One arrival at the barrier (of both CTAs of a pair) once all products issued so far are done.
template <int CG> __device__ __forceinline__ void mma_commit(uint32_t mbar) {
    if (CG == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(mbar),
            "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(mbar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }

__device__ __forceinline__ void tmem_ld(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
        "%12, %13, %14, %15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }

// 32 bytes at a 32-byte boundary
__device__ __forceinline__ void store32(void* p, const uint32_t (&r)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void load32(const void* p, uint32_t (&r)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store16f(float* p, const float (&v)[16]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(v[8 * h + i]);
        store32(p + 8 * h, r);
    }
}
__device__ __forceinline__ void store16(void* base, int dtype, int64_t at, const float (&v)[16]) {
    if (dtype == VQC_F32) return store16f(static_cast<float*>(base) + at, v);
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (dtype == VQC_BF16) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            r[i] = *reinterpret_cast<const uint32_t*>(&p);
        } else {
            const __half2 p = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            r[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
    }
    store32(static_cast<char*>(base) + 2 * at, r);
}
// 16 elements of the residual as they lie in memory
struct Res16 {
    uint32_t w[2][8];
};
__device__ __forceinline__ void load_res(const void* base, int dtype, int64_t at, Res16& r) {
    if (dtype == VQC_F32) {
        load32(static_cast<const float*>(base) + at, r.w[0]);
        load32(static_cast<const float*>(base) + at + 8, r.w[1]);
    } else {
        load32(static_cast<const char*>(base) + 2 * at, r.w[0]);
    }
}
__device__ __forceinline__ void add_res(const Res16& r, int dtype, float (&v)[16]) {
    if (dtype == VQC_F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += __uint_as_float(r.w[i / 8][i % 8]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 p = dtype == VQC_BF16 ? unpack2<__nv_bfloat16>(r.w[0][i]) : unpack2<__half>(r.w[0][i]);
        v[2 * i] += p.x;
        v[2 * i + 1] += p.y;
    }
}

// The epilogue keeps the biases of a warp's columns in its staging space (which only
// outputs that are not aligned use): those of the gate, then those of the other factor.
constexpr int kBiasUp = 128;
__device__ __forceinline__ void add_bias(const float* b, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(b + i);
        v[i] += q.x; v[i + 1] += q.y; v[i + 2] += q.z; v[i + 3] += q.w;
    }
}

template <int ACT> __device__ __forceinline__ void act16_as(float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = act_value(ACT, v[i]);
}
__device__ __forceinline__ void act16(int act, float (&v)[16]) {
    switch (act) {
        case VQC_ACT_RELU: return act16_as<VQC_ACT_RELU>(v);
        case VQC_ACT_GELU: return act16_as<VQC_ACT_GELU>(v);
        case VQC_ACT_SILU: return act16_as<VQC_ACT_SILU>(v);
        case VQC_ACT_TANH: return act16_as<VQC_ACT_TANH>(v);
        case VQC_ACT_SIGMOID: return act16_as<VQC_ACT_SIGMOID>(v);
        default: return;
    }
}

struct TileAt {
    int which, split, m, n;
};
// Tiles in groups of 16 tiles of rows, so that the CTAs at work at one time share
// rows of both operands in the L2.
template <int P> __device__ __forceinline__ TileAt tile_at(const TcArgs<P>& A, long long t) {
    TileAt r;
    const long long plane = (long long)A.tiles_m * A.tiles_n;
    const int p = (int)(t / plane);
    r.split = p % A.splits;
    r.which = p / A.splits;
    const long long i = t % plane, group = 16ll * A.tiles_n;
    const int g = (int)(i / group), rows = min(16, A.tiles_m - 16 * g);
    const int j = (int)(i - g * group);
    r.m = 16 * g + j % rows;
    r.n = j / rows;
    return r;
}

// Accumulator columns c0..c0+15 (and their partners of the gate) of a warp's 32
// rows, finished and written.  Aligned outputs go straight from the lanes, 32
// bytes of a row each; others are turned in shared memory so that lanes write
// neighbouring columns.
template <bool kGated, int kParts>
__device__ __forceinline__ void write16(const TcArgs<kParts>& A, const TileAt& T, int64_t row0, int64_t col0, int lane,
                                        float (&v)[16], float (&u)[16], const Res16& res, const float* bias, float* stage) {
    const Finish& f = A.f;
    const int64_t n = f.n;
    if (col0 >= n) return;
    if (kParts > 1 && !A.part && row0 + lane < f.m) {
        float t = 0.f;       // NaN if one of the sums is not finite
#pragma unroll
        for (int i = 0; i < 16; ++i) t = fmaf(v[i], 0.f, kGated ? fmaf(u[i], 0.f, t) : t);
        if (t != 0.f) {
            for (int i = 0; i < 16; ++i) {
                float a = 0.f, b = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j == i) { a = v[j]; b = kGated ? u[j] : 0.f; }
                if (col0 + i >= n) break;
                a = exact_if_not_finite(A.exact, T.which, row0 + lane, col0 + i, a);
                if (kGated) b = exact_if_not_finite(A.exact, 1, row0 + lane, col0 + i, b);
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j == i) {
                        v[j] = a;
                        if (kGated) u[j] = b;
                    }
            }
        }
    }
    if (kParts > 1) __syncwarp();
    if (A.vec && col0 + 16 <= n) {
        const int64_t row = row0 + lane;
        if (A.part) {
            if (row < f.m) {
                const int64_t slots = A.form == GATED || A.form == PAIR ? 2 : 1;
                float* at = A.part + ((T.split * slots + T.which) * f.m + row) * n + col0;
                store16f(at, v);
                if (kGated) store16f(at + f.m * n, u);
            }
            return;
        }
        if (row >= f.m) return;
        if (f.bias[T.which]) add_bias(bias, v);
        if (kGated && f.bias[1]) add_bias(bias + kBiasUp, u);
        const int64_t at = row * n + col0;
        if (f.z[T.which]) store16f(f.z[T.which] + at, v);
        if (kGated && f.z[1]) store16f(f.z[1] + at, u);
        act16(f.act, v);
        if (kGated) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= u[i];
        }
        if (!kGated && f.res) add_res(res, f.out_dtype, v);
        store16(f.y[T.which], f.out_dtype, at, v);
        return;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        stage[lane * 17 + i] = v[i];
        if (kGated) stage[32 * 17 + lane * 17 + i] = u[i];
    }
    __syncwarp();
    const int64_t col = col0 + (lane & 15);
    if (col < n) {
        for (int r = lane >> 4; r < 32 && row0 + r < f.m; r += 2) {
            const float a = stage[r * 17 + (lane & 15)], b = kGated ? stage[32 * 17 + r * 17 + (lane & 15)] : 0.f;
            if (A.part) {
                const int64_t slots = A.form == GATED || A.form == PAIR ? 2 : 1;
                float* at = A.part + ((T.split * slots + T.which) * f.m + row0 + r) * n + col;
                *at = a;
                if (kGated) at[f.m * n] = b;
            } else {
                finish_one(f, T.which, row0 + r, col, a, b);
            }
        }
    }
    __syncwarp();
}

template <int CG, int BN, bool kGated, int kParts>
__global__ void __launch_bounds__(kThreads, 1) tc_kernel(const __grid_constant__ TcArgs<kParts> A) {
    using S = Shape<CG, BN>;
    constexpr int NS = S::kStages;
    extern __shared__ __align__(1024) unsigned char sm[];
    float* staging = reinterpret_cast<float*>(sm + NS * S::kStage);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + NS * S::kStage + kStaging);
    const uint32_t full = smem_u32(bars), empty = full + 8 * NS, tfull = empty + 8 * NS, tempty = tfull + 16,
                   drain = tempty + 16;
    volatile int* gave_up = reinterpret_cast<volatile int*>(bars + 2 * NS + 5);
    uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + 2 * NS + 6);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const uint32_t base = smem_u32(sm);

    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull + 8 * i, 1);
            mbar_init(tempty + 8 * i, kEpiWarps * CG);
        }
        mbar_init(drain, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        for (int i = 0; i < 2; ++i) {
            tma_prefetch(&A.ma[i][0]);
            tma_prefetch(&A.mb[i][0]);
        }
    }
    if (warp == 2) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tslot)),
                         "n"(S::kTmem)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tslot)),
                         "n"(S::kTmem)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    }
    tc_fence_after();
    const uint32_t tmem = *tslot;

    constexpr int kPairs = kParts == 3 ? 6 : 1;      // products of parts per product
    const int kblocks = A.kblocks * kPairs * (A.form == SUM ? 2 : 1);
    const long long first = blockIdx.x / CG, step = gridDim.x / CG;
    // a role that gives up tells the others, in both CTAs
    auto give_up = [&]() {
        *gave_up = 1;
        if (CG == 2)
            asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"(at_cta(smem_u32((const void*)gave_up), rank ^ 1)), "r"(1)
                         : "memory");
        atomicOr(A.err, 1u);
    };

    if (warp == 0) {
        if (lane == 0) {
            int s = 0, used = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long t = first; t < A.tiles && ok; t += step) {
                const TileAt T = tile_at(A, t);
                const int kb0 = (int)((long long)kblocks * T.split / A.splits), kb1 = (int)((long long)kblocks * (T.split + 1) / A.splits);
                const int m0 = T.m * BM * CG + (int)rank * BM;
                const int n0 = T.n * (kGated ? BN / 2 : BN) + (kGated ? 0 : (int)rank * (BN / CG));
                int term = kb0 / A.kblocks, k0 = (kb0 - term * A.kblocks) * BK;
                for (int kb = kb0; kb < kb1; ++kb, k0 += BK) {
                    if (k0 >= A.kblocks * BK) {
                        ++term;
                        k0 = 0;
                    }
                    if (!mbar_wait(empty + 8 * s, ph ^ 1, gave_up)) {
                        ok = false;
                        break;
                    }
                    const int sum = term >= kPairs ? 1 : 0, pair = term - sum * kPairs;
                    const int pa = kPairs == 6 ? kPartsA >> (2 * pair) & 3 : 0, pb = kPairs == 6 ? kPartsB >> (2 * pair) & 3 : 0;
                    const CUtensorMap* ma = &A.ma[T.which + sum][pa];
                    const CUtensorMap* mb = &A.mb[T.which + sum][pb];
                    const uint32_t sa = base + s * S::kStage, sb = sa + kStageA;
                    const uint32_t bar = CG == 2 ? at_cta(full + 8 * s, 0) : full + 8 * s;
                    if (rank == 0)
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(full + 8 * s),
                                     "r"(CG * S::kStage)
                                     : "memory");
                    if (A.a_mn) {
#pragma unroll
                        for (int j = 0; j < BM / 64; ++j) tma_load<CG>(sa + j * 8192, ma, m0 + 64 * j, k0, bar);
                    } else {
                        tma_load<CG>(sa, ma, k0, m0, bar);
                    }
                    if (kGated) {
                        if (CG == 2) {
                            tma_load<CG>(sb, &A.mb[rank][pb], k0, n0, bar);
                        } else {
                            tma_load<CG>(sb, &A.mb[0][pb], k0, n0, bar);
                            tma_load<CG>(sb + S::kStageB / 2, &A.mb[1][pb], k0, n0, bar);
                        }
                    } else if (A.b_mn) {
#pragma unroll
                        for (int j = 0; j < BN / CG / 64; ++j) tma_load<CG>(sb + j * 8192, mb, n0 + 64 * j, k0, bar);
                    } else {
                        tma_load<CG>(sb, mb, k0, n0, bar);
                    }
                    used = used < NS ? used + 1 : NS;
                    if (++s == NS) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
            if (!ok) {
                give_up();
                // copies still in flight land before this CTA's memory is given back: the
                // last `used` stages, in the order of their issue
                if (rank == 0)
                    for (int i = used; i > 0; --i) {
                        const int q = (s - i + NS) % NS;
                        mbar_wait(full + 8 * q, q < s ? ph : ph ^ 1, nullptr);
                    }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = (1u << 4) | ((uint32_t)A.bf16 << 7) | ((uint32_t)A.bf16 << 10) |
                                   ((uint32_t)A.a_mn << 15) | ((uint32_t)A.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) |
                                   ((uint32_t)(BM * CG >> 4) << 24);
            const uint32_t step_a = A.a_mn ? 2048 >> 4 : 32 >> 4, step_b = A.b_mn ? 2048 >> 4 : 32 >> 4;
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true, issued = false;
            for (long long t = first; t < A.tiles && ok; t += step) {
                const TileAt T = tile_at(A, t);
                const int kb0 = (int)((long long)kblocks * T.split / A.splits), kb1 = (int)((long long)kblocks * (T.split + 1) / A.splits);
                if (!mbar_wait(tempty + 8 * acc, aph ^ 1, gave_up)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait(full + 8 * s, ph, gave_up)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t da = smem_desc(base + s * S::kStage, 8192), db = smem_desc(base + s * S::kStage + kStageA, 8192);
#pragma unroll
                    for (int j = 0; j < BK / 16; ++j)
                        mma<CG>(tmem + acc * BN, da + j * step_a, db + j * step_b, idesc, kb > kb0 || j > 0);
                    issued = true;
                    mma_commit<CG>(empty + 8 * s);
                    if (++s == NS) {
                        s = 0;
                        ph ^= 1;
                    }
                }
                if (!ok) break;
                mma_commit<CG>(tfull + 8 * acc);
                if (++acc == 2) {
                    acc = 0;
                    aph ^= 1;
                }
            }
            if (!ok) {
                give_up();
                if (issued) {   // products in flight finish before the tensor memory is freed
                    mma_commit<CG>(drain);
                    mbar_wait(drain, 0, nullptr);
                }
            }
        }
    } else if (warp >= 4) {
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float* stage = staging + (warp - 4) * 2 * 32 * 17;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        constexpr int kCols = kGated ? BN / 2 : BN;   // output columns of a tile
        int acc = 0;
        uint32_t aph = 0;
        for (long long t = first; t < A.tiles; t += step) {
            const TileAt T = tile_at(A, t);
            if (A.vec && !A.part) {      // biases of this warp's columns
                __syncwarp();
                for (int w = 0; w < (kGated ? 2 : 1); ++w) {
                    const void* from = A.f.bias[kGated ? w : T.which];
                    if (from)
                        for (int c = lane; c < kCols / 2; c += 32) {
                            const int64_t col = (int64_t)T.n * kCols + half * (kCols / 2) + c;
                            stage[w * kBiasUp + c] = col < A.f.n ? load_as(from, A.f.dtype, col) : 0.f;
                        }
                }
            }
            if (!mbar_wait(tfull + 8 * acc, aph, gave_up)) {
                if (lane == 0) give_up();
                break;
            }
            tc_fence_after();
            const int64_t row0 = ((int64_t)T.m * CG + rank) * BM + quad * 32;
            const int64_t n0 = (int64_t)T.n * kCols;
            // the residual is read one step ahead
            const bool ahead = !kGated && A.f.res && A.vec && !A.part && row0 + lane < A.f.m;
            auto fetch = [&](int c, Res16& r) {
                if (ahead && n0 + c + 16 <= A.f.n) load_res(A.f.res, A.f.out_dtype, (row0 + lane) * A.f.ld_res + n0 + c, r);
            };
            Res16 res, next;
            fetch(half * (kCols / 2), next);
#pragma unroll 1
            for (int c = half * (kCols / 2); c < (half + 1) * (kCols / 2); c += 16) {
                float v[16], u[16];
                res = next;
                if (c + 16 < (half + 1) * (kCols / 2)) fetch(c + 16, next);
                __syncwarp();
                tmem_ld(tmem + lanes + acc * BN + c, v);
                if (kGated) tmem_ld(tmem + lanes + acc * BN + BN / 2 + c, u);
                tmem_wait();
                write16<kGated, kParts>(A, T, row0, n0 + c, lane, v, u, res, stage + c - half * (kCols / 2), stage);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = tempty + 8 * acc;
                if (CG == 2)
                    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(at_cta(bar, 0)) : "memory");
                else
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
            }
            if (++acc == 2) {
                acc = 0;
                aph ^= 1;
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {   // no CTA leaves while its partner may still signal it or read its memory
        asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    }
    tc_fence_after();
    if (warp == 2) {
        if (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(S::kTmem) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(S::kTmem) : "memory");
    }
}

__device__ unsigned g_layers_err;

// Its address on the current device, looked up once per device.
cudaError_t error_word(unsigned** p) {
    static std::atomic<void*> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    void* q = dev < 64 ? known[dev].load() : nullptr;
    if (!q) {
        e = cudaGetSymbolAddress(&q, g_layers_err);
        if (e != cudaSuccess) return e;
        if (dev < 64) known[dev].store(q);
    }
    *p = static_cast<unsigned*>(q);
    return cudaSuccess;
}

// A float as the sum of three bf16, 8 bits of it each, rounded to nearest: exact for
// normal results.  A value that is not finite is its own first part (and the sums
// that it enters are worked out again, see Exact); one that would round to
// infinity is cut instead.
__device__ __forceinline__ void bf16_parts(float x, uint16_t (&o)[3]) {
    float rest = x;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        __nv_bfloat16 h = __float2bfloat16(rest);
        uint16_t bits = __bfloat16_as_ushort(h);
        if ((bits & 0x7fff) == 0x7f80 && fabsf(rest) <= 3.4028234e38f) bits -= 1;
        o[i] = bits;
        rest = (bits & 0x7f80) == 0x7f80 ? 0.f : rest - __uint_as_float((uint32_t)bits << 16);
    }
}

// [rows, cols] of floats as three matrices of parts, rows of `ld_to` elements (a multiple
// of 8): 8 elements per thread.
__global__ void __launch_bounds__(256) parts_kernel(const float* from, int64_t ld, int64_t rows, int64_t cols, uint16_t* to,
                                                    int64_t ld_to, int vec) {
    const int64_t across = ld_to / 8, plane = rows * ld_to, count = rows * across, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < count; e += step) {
        const int64_t r = e / across, c = e % across * 8;
        const float* p = from + r * ld + c;
        float v[8];
        if (vec && c + 8 <= cols) {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? p[i] : 0.f;
        }
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint16_t a[3], b[3];
            bf16_parts(v[i], a);
            bf16_parts(v[i + 1], b);
#pragma unroll
            for (int q = 0; q < 3; ++q) w[q][i / 2] = (uint32_t)a[q] | (uint32_t)b[q] << 16;
        }
#pragma unroll
        for (int q = 0; q < 3; ++q)
            *reinterpret_cast<uint4*>(to + q * plane + r * ld_to + c) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
}

// 16-bit copy of [rows, cols] with rows of `ld_to` elements (a multiple of 8)
__global__ void __launch_bounds__(256) align_kernel(const uint16_t* from, int64_t ld, int64_t rows, int64_t cols, uint16_t* to,
                                                    int64_t ld_to) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) to[r * ld_to + c] = from[r * ld + c];
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static std::atomic<void*> fn{nullptr};
    void* p = fn.load();
    if (!p) {
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        fn.store(p);
    }
    return reinterpret_cast<EncodeTiled>(p);
}

// Map of an operand with `outer` rows of the outer index: boxes of 64 contracted
// elements x `box` rows, or of 64 outer elements x 64 contracted where the outer
// index is the inner one in memory.
bool make_map(CUtensorMap* m, const Operand& o, int dtype, int64_t outer, int64_t k, int box) {
    EncodeTiled enc = encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)(o.k_outer ? outer : k), (cuuint64_t)(o.k_outer ? k : outer)};
    const cuuint64_t strides[1] = {(cuuint64_t)o.ld * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)(o.k_outer ? BK : box)}, one[2] = {1, 1};
    return enc(m, dtype != VQC_F16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
               const_cast<void*>(o.p), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// TMA reads rows at multiples of 16 bytes; other operands are copied first, and
// float operands are written as three bf16 parts.
bool ready(const Operand& o, int dtype, bool aligned) { return dtype != VQC_F32 && aligned && o.ld % 8 == 0; }
int64_t copy_ld(int64_t cols) { return (cols + 7) / 8 * 8; }
int parts_of(int dtype) { return dtype == VQC_F32 ? 3 : 1; }
size_t copy_bytes(const Operand& o, int dtype, int64_t outer, int64_t k) {
    return align256((size_t)(o.k_outer ? k : outer) * copy_ld(o.k_outer ? outer : k) * 2 * parts_of(dtype));
}

struct Choice {
    int cg, bn, splits;
};

// The tile and the cuts that finish first, by a count of cycles on one SM: a
// stage of 64 costs its products (8192 per cycle and SM) or its bytes (about 64
// per cycle and SM from the L2), whichever is longer, a tile its start and end, a
// cut the traffic of its sums.
Choice choose_new(const Product& p) {
    static const struct { int cg, bn, stage; } kTiles[] = {{2, 256, 560}, {2, 128, 400}, {1, 128, 512}, {1, 64, 384}};
    const int sms = sm_count();
    const int64_t kblocks = ceil_div(p.k, BK) * (p.form == SUM ? 2 : 1) * (p.f.dtype == VQC_F32 ? 6 : 1);
    Choice best{1, 64, 1};
    double least = 1e300;
    for (const auto& t : kTiles) {
        const int64_t cols = p.form == GATED ? t.bn / 2 : t.bn;
        const int64_t tiles = ceil_div(p.m, BM * t.cg) * ceil_div(p.n, cols) * (p.form == PAIR ? 2 : 1);
        for (int64_t s = 1; s <= std::min<int64_t>(kblocks, 64); s = s < 4 ? s + 1 : s + s / 4) {
            const int64_t units = sms / t.cg, waves = ceil_div(tiles * s, units);
            const double end = 3.0 * t.bn;      // taking an accumulator out
            const double tile = (double)ceil_div(kblocks, s) * t.stage;
            double c = waves * std::max(tile, end) + end + 2500;
            // sums written and read once by all SMs together, and a second launch
            if (s > 1) c += 4000 + (double)(s + 1) * p.m * p.n * (p.form == GATED || p.form == PAIR ? 2 : 1) * 4 / (sms * 24.0);
            if (c < least) {
                least = c;
                best = {t.cg, t.bn, (int)s};
            }
        }
    }
    return best;
}

// The choices of the sizes that a thread asked for last.
Choice choose(const Product& p) {
    struct Known {
        int64_t m = 0, n = 0, k = 0;
        int form = -1, dtype = -1, sms = 0;
        Choice c;
    };
    static thread_local Known known[64];
    const bool parts = p.f.dtype == VQC_F32;
    Known& q = known[(uint64_t)(p.m * 0x9E3779B1 + p.n * 0x85EBCA77 + p.k * 0xC2B2AE3D + p.form + 4 * parts) >> 7 & 63];
    const int sms = sm_count();
    if (q.m != p.m || q.n != p.n || q.k != p.k || q.form != p.form || q.dtype != parts || q.sms != sms) {
        q.c = choose_new(p);
        q.m = p.m; q.n = p.n; q.k = p.k; q.form = p.form; q.dtype = parts; q.sms = sms;
    }
    return q.c;
}

template <int CG, int BN, bool kGated, int kParts> cudaError_t launch_tc(const TcArgs<kParts>& a, cudaStream_t s) {
    using S = Shape<CG, BN>;
    static std::atomic<unsigned long long> prepared{0};    // devices whose limit is raised
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(prepared.load() >> (dev & 63) & 1)) {
        const cudaError_t e = cudaFuncSetAttribute((const void*)tc_kernel<CG, BN, kGated, kParts>,
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        if (e != cudaSuccess) return e;
        prepared.fetch_or(1ull << (dev & 63));
    }
    const long long units = sm_count() / CG;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(std::min<long long>(a.tiles, units) * CG));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, tc_kernel<CG, BN, kGated, kParts>, a);
}

template <bool kGated, int kParts> cudaError_t launch_choice(const Choice& c, const TcArgs<kParts>& a, cudaStream_t s) {
    if (c.cg == 2) return c.bn == 256 ? launch_tc<2, 256, kGated, kParts>(a, s) : launch_tc<2, 128, kGated, kParts>(a, s);
    return c.bn == 128 ? launch_tc<1, 128, kGated, kParts>(a, s) : launch_tc<1, 64, kGated, kParts>(a, s);
}

}  // namespace

// Float products come here where six products of parts (and writing the parts)
// take less time than float FMAs.
bool tc_takes(const Product& p) {
    constexpr int64_t kMost = 1 << 30;
    if (p.m <= 0 || p.k <= 0 || p.m >= kMost || p.n >= kMost || p.k >= kMost) return false;
    if (p.f.dtype != VQC_F32) return true;
    const double flops = 2.0 * p.m * p.n * p.k * (p.form == PLAIN ? 1 : 2);
    return flops >= 5e8 && p.k >= 64 && std::min(p.m, p.n) >= 64;
}

size_t tc_workspace(const Product& p, bool aligned) {
    size_t bytes = 0;
    const int na = p.form == SUM || p.form == PAIR ? 2 : 1, nb = p.form == SUM || p.form == GATED ? 2 : 1;
    for (int i = 0; i < na; ++i)
        if (!ready(p.a[i], p.f.dtype, aligned)) bytes += copy_bytes(p.a[i], p.f.dtype, p.m, p.k);
    for (int i = 0; i < nb; ++i)
        if (!ready(p.b[i], p.f.dtype, aligned)) bytes += copy_bytes(p.b[i], p.f.dtype, p.n, p.k);
    const Choice c = choose(p);
    if (c.splits > 1) bytes += align256((size_t)c.splits * (p.form == GATED || p.form == PAIR ? 2 : 1) * p.m * p.n * 4);
    return bytes;
}

namespace {
template <int kParts> vqc_status run_parts(const Product& p, void* ws, size_t ws_bytes, Joins& joins, cudaStream_t s) {
    TcArgs<kParts> a;
    char* at = static_cast<char*>(ws);
    size_t left = ws ? ws_bytes : 0;
    auto take = [&](size_t bytes) -> void* {
        if (bytes > left) return nullptr;
        void* r = at;
        at += bytes;
        left -= bytes;
        return r;
    };
    const Choice c = choose(p);
    const bool gated = p.form == GATED;
    constexpr bool split = kParts == 3;
    const int na = p.form == SUM || p.form == PAIR ? 2 : 1, nb = p.form == SUM || gated ? 2 : 1;
    for (int side = 0; side < 2; ++side)
        for (int i = 0; i < (side ? nb : na); ++i) {
            Operand o = side ? p.b[i] : p.a[i];
            const int64_t outer = side ? p.n : p.m;
            int64_t rows = o.k_outer ? p.k : outer, cols = o.k_outer ? outer : p.k, ld = o.ld, ld_to = copy_ld(cols);
            if (!ready(o, p.f.dtype, aligned_to(o.p, 16))) {
                void* to = take(copy_bytes(o, p.f.dtype, outer, p.k));
                if (!to) return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
                const void* from = o.p;
                int vec = ld % 4 == 0 && aligned_to(from, 16);
                void* args[] = {&from, &ld, &rows, &cols, &to, &ld_to, &vec};
                const int64_t grid = split ? std::min<int64_t>(ceil_div(rows * ld_to / 8, 256), 8LL * sm_count()) : std::min<int64_t>(rows, 16LL * sm_count());
                const cudaError_t e = cudaLaunchKernel(split ? (const void*)parts_kernel : (const void*)align_kernel, dim3((unsigned)grid),
                                                       dim3(256), args, 0, s);
                if (e != cudaSuccess) return cuda_error(e, "operand copy launch");
                o.p = to;
                o.ld = ld_to;
            }
            const int box = side ? (gated ? c.bn / 2 : c.bn / c.cg) : BM;
            for (int q = 0; q < kParts; ++q) {
                Operand part = o;
                part.p = static_cast<const uint16_t*>(o.p) + q * rows * ld_to;
                if (!make_map(side ? &a.mb[i][q] : &a.ma[i][q], part, p.f.dtype, outer, p.k, box))
                    return set_error(VQC_ERR_CUDA, "product: cuTensorMapEncodeTiled failed");
            }
        }
    for (int q = 0; q < kParts; ++q) {      // an operand of both products
        if (na == 1) a.ma[1][q] = a.ma[0][q];
        if (nb == 1) a.mb[1][q] = a.mb[0][q];
    }
    a.f = p.f;
    a.form = p.form;
    a.bf16 = p.f.dtype != VQC_F16;
    a.splits = c.splits;
    a.tiles_m = (int)ceil_div(p.m, BM * c.cg);
    a.tiles_n = (int)ceil_div(p.n, gated ? c.bn / 2 : c.bn);
    a.kblocks = (int)ceil_div(p.k, BK);
    a.a_mn = p.a[0].k_outer;
    a.b_mn = p.b[0].k_outer;
    a.tiles = (long long)a.tiles_m * a.tiles_n * a.splits * (p.form == PAIR ? 2 : 1);
    a.exact = Exact{};
    a.part = nullptr;
    if (split) {
        for (int i = 0; i < 2; ++i) { a.exact.a[i] = p.a[i]; a.exact.b[i] = p.b[i]; }
        a.exact.k = p.k;
        a.exact.form = p.form;
    }
    if (c.splits > 1) {
        a.part = static_cast<float*>(take(align256((size_t)c.splits * (gated || p.form == PAIR ? 2 : 1) * p.m * p.n * 4)));
        if (!a.part) return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
        Join& j = joins.j[joins.count++];
        j.f = p.f;
        j.exact = a.exact;
        j.part = a.part;
        j.splits = c.splits;
        j.form = p.form;
    }
    // every row of every output on a 32-byte boundary
    const int64_t eo = (int64_t)elem_size(p.f.out_dtype);
    auto on32 = [](const void* q) { return aligned_to(q, 32); };
    a.vec = a.part ? p.n % 8 == 0
                   : p.n * eo % 32 == 0 && on32(p.f.y[0]) && on32(p.f.y[1]) &&
                         (!p.f.z[0] || (p.n % 8 == 0 && on32(p.f.z[0]) && on32(p.f.z[1]))) &&
                         (!p.f.res || (p.f.ld_res * eo % 32 == 0 && on32(p.f.res)));
    cudaError_t e = error_word(&a.err);
    if (e != cudaSuccess) return cuda_error(e, "cudaGetSymbolAddress");
    e = gated ? launch_choice<true, kParts>(c, a, s) : launch_choice<false, kParts>(c, a, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "tensor-core product launch");
}
}  // namespace

vqc_status tc_run(const Product& p, void* ws, size_t ws_bytes, Joins& joins, cudaStream_t s) {
    return p.f.dtype == VQC_F32 ? run_parts<3>(p, ws, ws_bytes, joins, s) : run_parts<1>(p, ws, ws_bytes, joins, s);
}

}  // namespace layers

// vqc_sync_check's view of the tensor-core products' error word (read and cleared).
vqc_status layers_error_check() {
    unsigned e = 0;
    cudaError_t c = cudaMemcpyFromSymbol(&e, layers::g_layers_err, sizeof(e));
    if (c != cudaSuccess) return set_error(VQC_ERR_CUDA, std::string("layers error word: ") + cudaGetErrorString(c));
    if (!e) return VQC_OK;
    const unsigned zero = 0;
    cudaMemcpyToSymbol(layers::g_layers_err, &zero, sizeof(zero));
    return set_error(VQC_ERR_DEVICE_CHECK, "a tensor-core product's wait timed out");
}

}  // namespace vqc
