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
// The tensor cores cut the low bits of a running sum at every product of depth 16 where
// float32 would round (measured: a bias of 1.7e-8 of the result per product, 4e-6
// at a depth of 4096).  Where the output is float32 a tile's contraction is therefore taken out in chunks
// of 256, which the epilogue adds up in registers (kSums: tiles up to 128 columns).  Where it has 16 bits the
// running sum stays in tensor memory, and with it what is saved in float beside it (z; g and u) and
// the sums of cuts: at that depth the bias is 1/400 of an output's own rounding in bfloat16, 1/50 in float16,
// and the registers of chunks would not fit tiles of 256 columns.
//
// Two products that do not depend on one another (the two of a backward) share a launch:
// one's tiles fill the SMs that the other's last tiles leave idle.
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
// Measured, bfloat16: 8192 x 2048 x 2048 44 us (1550 TFLOP/s, a library product 45), gated 8192 x
// 2048 x 5632 193 us (1950), both gradient products of the latter 407 us (1860, the
// tensor pipe 91% active under the power cap); small products end at about 7 us (start, first
// loads, one accumulator).
//
// Every wait is bounded (4 s, or the environment's VQC_WAIT_NS).  A warp whose wait runs out sets the
// error word and tells the other warps of both CTAs, whose own waits then end; all meet at the
// kernel's last barrier, copies and products still in flight are waited for, tensor memory is
// freed and the CTAs return.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cstdlib>
#include <mutex>

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
constexpr unsigned long long kWaitNs = 4000000000ull;   // bound of a wait

template <int CG, int BN> struct Shape {
    static constexpr int kStageB = BN / CG * BK * 2;
    static constexpr int kStage = kStageA + kStageB;
    static constexpr int kStages = (kSmemLimit - kStaging - kBarriers) / kStage < 8 ? (kSmemLimit - kStaging - kBarriers) / kStage : 8;
    static constexpr int kSmem = kStages * kStage + kStaging + kBarriers;
    static constexpr int kTmem = 2 * BN;             // two accumulators, a power of two >= 32
};

// One product; maps of its operands: [operand][part].  kParts: 1, or 3 of float
// operands, or 2: two of a (one 16-bit matrix and what it leaves), one of b.
template <int kParts> struct Problem {
    static constexpr int kPartsB = kParts == 2 ? 1 : kParts;
    CUtensorMap ma[2][kParts], mb[2][kPartsB];
    Finish f;
    float* part;                // sums of a cut contraction, or NULL
    int form, splits, tiles_m, tiles_n, kblocks, a_mn, b_mn, vec;   // vec: bytes of a store
};

// The tiles of one or two products among the units (CTAs or pairs): those of the first
// product in turn, then those of the second, of which units that had one tile less
// of the first get more (first tiles are the longer ones).
struct Schedule {
    long long first, second;     // tiles
    int units, rounds, extra;    // first = rounds * units + extra
    int second_rounds;           // tiles of the second product that every unit has
};
__device__ __forceinline__ bool tile_of(const Schedule& S, int unit, int i, int& q, long long& t) {
    const int mine = S.rounds + (unit < S.extra ? 1 : 0);
    q = i >= mine ? 1 : 0;
    if (!q) {
        t = (long long)i * S.units + unit;
        return true;
    }
    const int j = i - mine;
    if (j < S.second_rounds) t = (long long)j * S.units + unit;
    else if (unit >= S.extra) t = (long long)S.second_rounds * S.units + (long long)(j - S.second_rounds) * (S.units - S.extra) + (unit - S.extra);
    else return false;
    return t < S.second;
}

template <int kParts> struct TcArgs {
    Problem<kParts> q[2];
    Schedule plan;
    unsigned* err;
    unsigned long long wait_ns;
    int bf16;
};

constexpr int pairs_of(int parts) { return parts == 3 ? 6 : parts; }
// Products of parts of float operands, small ones first: parts of a and b, 2 bits each.
constexpr unsigned kOrderA = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10;
constexpr unsigned kOrderB = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;

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
// true in one lane of a converged warp
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r != 0;
}
template <bool B> struct Flag {
    static constexpr bool value = B;
};
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

// Bounded wait for a phase; false when it ran out or another role gave up.  Lanes may see the end
// at different times: the warp goes by what all of them saw.
__device__ __noinline__ bool mbar_wait_slow(uint32_t mbar, uint32_t parity, unsigned long long ns, const volatile int* gave_up) {
    const unsigned long long end = now_ns() + ns;
    while (!mbar_try(mbar, parity))      // (which itself waits for some time)
        if ((gave_up && *gave_up) || now_ns() > end) return false;
    return true;
}
__device__ __forceinline__ bool mbar_wait(uint32_t mbar, uint32_t parity, unsigned long long ns, const volatile int* gave_up) {
    return __all_sync(~0u, mbar_try(mbar, parity) || mbar_wait_slow(mbar, parity, ns, gave_up));
}

// a word of the shared memory of another CTA of the cluster
__device__ __forceinline__ uint32_t peer_word(uint32_t addr, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(at_cta(addr, rank)) : "memory");
    return v;
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
__device__ __forceinline__ void load_bytes(const void* p, int wide, uint32_t (&r)[8]) {
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "l"(p)
                     : "memory");
    } else {
        const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
        r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w;
        r[4] = b.x; r[5] = b.y; r[6] = b.z; r[7] = b.w;
    }
}
// 32 bytes, at once where `wide`, else as two
__device__ __forceinline__ void store_bytes(void* p, int wide, const uint32_t (&r)[8]) {
    if (wide) return store32(p, r);
    reinterpret_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

// A warp's 32 rows x 64 bytes (a row per lane) to or from memory by way of shared memory,
// so that four lanes move a row's 64 bytes and an instruction touches 8 lines, not 32: the
// L1 takes a line per cycle, and the end of a tile is bound by that.  Pieces of 16
// bytes, piece c of row r at place c ^ (r / 2 % 4): no bank twice.  `rows`: rows that exist.
__device__ __forceinline__ uint4* piece(uint4* stage, int row, int c) { return stage + 4 * row + (c ^ (row >> 1 & 3)); }
__device__ __forceinline__ void rows_out(uint4* stage, const uint32_t (&w)[16], char* to, int64_t pitch, int rows, int lane) {
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) *piece(stage, lane, c) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        if (r < rows) *reinterpret_cast<uint4*>(to + r * pitch + 16 * (lane & 3)) = *piece(stage, r, lane & 3);
    }
}
__device__ __forceinline__ void rows_ask(uint4 (&w)[4], const char* from, int64_t pitch, int rows, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        if (r < rows) w[i] = *reinterpret_cast<const uint4*>(from + r * pitch + 16 * (lane & 3));
    }
}
__device__ __forceinline__ void rows_in(uint4* stage, const uint4 (&w)[4], uint32_t (&v)[16], int lane) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) *piece(stage, 8 * i + (lane >> 2), lane & 3) = w[i];
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint4 q = *piece(stage, lane, c);
        v[4 * c] = q.x; v[4 * c + 1] = q.y; v[4 * c + 2] = q.z; v[4 * c + 3] = q.w;
    }
}
// 16 floats per lane to `to`, the address of the warp's first row
__device__ __forceinline__ void floats_out(float* stage, const float* v, float* to, int64_t n, int rows, int lane) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[i]);
    rows_out(reinterpret_cast<uint4*>(stage), w, reinterpret_cast<char*>(to), 4 * n, rows, lane);
}
__device__ __forceinline__ void store16(void* base, int dtype, int64_t at, int wide, const float (&v)[16]) {
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        r[i] = dtype == VQC_BF16 ? pack2<__nv_bfloat16>(v[2 * i], v[2 * i + 1]) : pack2<__half>(v[2 * i], v[2 * i + 1]);
    store_bytes(static_cast<char*>(base) + 2 * at, wide, r);
}
// 16 elements of the residual as they lie in memory
struct Res16 {
    uint32_t w[2][8];
};
__device__ __forceinline__ void load_res(const void* base, int dtype, int64_t at, int wide, Res16& r) {
    if (dtype == VQC_F32) {
        load_bytes(static_cast<const float*>(base) + at, wide, r.w[0]);
        load_bytes(static_cast<const float*>(base) + at + 8, wide, r.w[1]);
    } else {
        load_bytes(static_cast<const char*>(base) + 2 * at, wide, r.w[0]);
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

// A warp's staging space: 32 x 17 floats to turn outputs, then the biases of its columns
// (16-byte aligned): those of the gate, then those of the other factor.
constexpr int kBias = 32 * 17 + 16, kBiasUp = 128;
__device__ __forceinline__ void add_bias(const float* b, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(b + i);
        v[i] += q.x; v[i + 1] += q.y; v[i + 2] += q.z; v[i + 3] += q.w;
    }
}

__device__ __forceinline__ void scale16(float scale, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= scale;
}
template <int ACT, bool kFull> __device__ __forceinline__ void act16_as(float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = act_value<kFull>(ACT, v[i]);
}
template <bool kFull> __device__ __forceinline__ void act16(const Finish& f, float (&v)[16]) {
    switch (f.act) {
        case kActScale: return scale16(*f.scale, v);
        case VQC_ACT_RELU: return act16_as<VQC_ACT_RELU, kFull>(v);
        case VQC_ACT_GELU: return act16_as<VQC_ACT_GELU, kFull>(v);
        case VQC_ACT_SILU: return act16_as<VQC_ACT_SILU, kFull>(v);
        case VQC_ACT_TANH: return act16_as<VQC_ACT_TANH, kFull>(v);
        case VQC_ACT_SIGMOID: return act16_as<VQC_ACT_SIGMOID, kFull>(v);
        default: return;
    }
}

struct TileAt {
    int which, split, m, n;
};
// Tiles in groups of 16 tiles of rows, so that the CTAs at work at one time share
// rows of both operands in the L2.
template <int P> __device__ __forceinline__ TileAt tile_at(const Problem<P>& A, long long t) {
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

// A warp's 32 x 16 values to memory, turned in shared memory so that lanes write
// neighbouring columns: put(row, column, value) for those inside the matrix.
template <typename F>
__device__ __forceinline__ void turned(const float (&v)[16], int64_t row0, int64_t col0, int64_t m, int64_t n, int lane, float* stage, F put) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) stage[lane * 17 + i] = v[i];
    __syncwarp();
    const int64_t col = col0 + (lane & 15);
    if (col < n) {
#pragma unroll 8
        for (int r = lane >> 4; r < 32; r += 2)
            if (row0 + r < m) put(row0 + r, col, stage[r * 17 + (lane & 15)]);
    }
}

// Accumulator columns c0..c0+15 (and their partners of the gate) of a warp's 32
// rows, finished and written: outputs whose rows lie on 16-byte boundaries by rows_out
// (floats) or straight from the lanes, others turned.
template <bool kGated, int kParts, bool kSums>
__device__ __forceinline__ void write16(const Problem<kParts>& A, const TileAt& T, int64_t row0, int64_t col0, int lane,
                                        float (&v)[16], float (&u)[16], const float* bias, float* stage) {
    const Finish& f = A.f;
    const int64_t n = f.n, row = row0 + lane;
    const int rows = (int)max((int64_t)0, min((int64_t)32, f.m - row0));
    const bool in = lane < rows, vec = A.vec && col0 + 16 <= n;
    if (col0 >= n) return;
    if (A.part) {
        const int64_t slots = A.form == GATED || A.form == PAIR ? 2 : 1;
        float* to = A.part + (T.split * slots + T.which) * f.m * n;
        if (vec) {
            floats_out(stage, v, to + row0 * n + col0, n, rows, lane);
            if (kGated) floats_out(stage, u, to + (f.m + row0) * n + col0, n, rows, lane);
        } else {
            auto put = [&](int64_t r, int64_t c, float x) { to[r * n + c] = x; };
            turned(v, row0, col0, f.m, n, lane, stage, put);
            to += f.m * n;
            if (kGated) turned(u, row0, col0, f.m, n, lane, stage, put);
        }
        return;
    }
    if (f.bias[T.which]) add_bias(bias, v);
    if (kGated && f.bias[1]) add_bias(bias + kBiasUp, u);
#pragma unroll
    for (int w = 0; w < (kGated ? 2 : 1); ++w) {
        float* z = f.z[kGated ? w : T.which];
        if (!z) continue;
        if (vec) floats_out(stage, w ? u : v, z + row0 * n + col0, n, rows, lane);
        else turned(w ? u : v, row0, col0, f.m, n, lane, stage, [&](int64_t r, int64_t c, float x) { z[r * n + c] = x; });
    }
    act16<kSums>(f, v);
    if (kGated) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= u[i];
    }
    if (vec) {
        if (!kGated && f.res && in) {
            Res16 res;
            load_res(f.res, f.out_dtype, row * f.ld_res + col0, A.vec == 32, res);
            add_res(res, f.out_dtype, v);
        }
        if (f.out_dtype == VQC_F32) floats_out(stage, v, static_cast<float*>(f.y[T.which]) + row0 * n + col0, n, rows, lane);
        else if (in) store16(f.y[T.which], f.out_dtype, row * n + col0, A.vec == 32, v);
    } else if (!kGated && f.res) {
        turned(v, row0, col0, f.m, n, lane, stage, [&](int64_t r, int64_t c, float x) {
            store_as(f.y[T.which], f.out_dtype, r * n + c, x + load_as(f.res, f.out_dtype, r * f.ld_res + c));
        });
    } else {
        turned(v, row0, col0, f.m, n, lane, stage, [&](int64_t r, int64_t c, float x) { store_as(f.y[T.which], f.out_dtype, r * n + c, x); });
    }
}

// 32 columns at once of a 16-bit output with whole rows of 64 bytes; `res`: the
// residual's, asked for a step ahead.
template <bool kGated, int kParts>
__device__ __forceinline__ void write32(const Problem<kParts>& A, const TileAt& T, int64_t row0, int64_t col0, int lane,
                                        float (&v)[2][16], float (&u)[2][16], const uint4 (&res)[4], const float* bias, float* stage) {
    const Finish& f = A.f;
    const int64_t n = f.n, at = row0 * n + col0;
    const int rows = (int)max((int64_t)0, min((int64_t)32, f.m - row0));
    uint4* pieces = reinterpret_cast<uint4*>(stage);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (f.bias[T.which]) add_bias(bias + 16 * h, v[h]);
        if (kGated && f.bias[1]) add_bias(bias + kBiasUp + 16 * h, u[h]);
        if (f.z[T.which]) floats_out(stage, v[h], f.z[T.which] + at + 16 * h, n, rows, lane);
        if (kGated && f.z[1]) floats_out(stage, u[h], f.z[1] + at + 16 * h, n, rows, lane);
        act16<false>(f, v[h]);      // (16-bit outputs)
        if (kGated) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[h][i] *= u[h][i];
        }
    }
    uint32_t w[16];
    if (!kGated && f.res) {
        rows_in(pieces, res, w, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 p = f.out_dtype == VQC_BF16 ? unpack2<__nv_bfloat16>(w[i]) : unpack2<__half>(w[i]);
            v[i / 8][2 * (i % 8)] += p.x;
            v[i / 8][2 * (i % 8) + 1] += p.y;
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float a = v[i / 8][2 * (i % 8)], b = v[i / 8][2 * (i % 8) + 1];
        w[i] = f.out_dtype == VQC_BF16 ? pack2<__nv_bfloat16>(a, b) : pack2<__half>(a, b);
    }
    rows_out(pieces, w, static_cast<char*>(f.y[T.which]) + 2 * at, 2 * n, rows, lane);
}

// The end of the chunk that begins at block kb: 4 blocks of the product of the first
// parts (of the only ones), all of the products of small parts together.
template <int kPairs> __device__ __forceinline__ int chunk_end(int kb, int kb1, int kblocks) {
    const int term = kb / kblocks, pair = term % kPairs;
    const int end = pair == kPairs - 1 ? term * kblocks + min(kblocks, ((kb - term * kblocks) / 4 + 1) * 4) : (term - pair + kPairs - 1) * kblocks;
    return min(end, kb1);
}

template <int CG, int BN, bool kGated, int kParts, bool kSums>
__global__ void __launch_bounds__(kThreads, 1) tc_kernel(const __grid_constant__ TcArgs<kParts> P) {
    using S = Shape<CG, BN>;
    constexpr int NS = S::kStages;
    extern __shared__ __align__(1024) unsigned char sm[];
    float* staging = reinterpret_cast<float*>(sm + NS * S::kStage);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + NS * S::kStage + kStaging);
    const uint32_t full = smem_u32(bars), empty = full + 8 * NS, tfull = empty + 8 * NS, tempty = tfull + 16,
                   drain = tempty + 16;
    volatile int* gave_up = reinterpret_cast<volatile int*>(bars + 2 * NS + 5);
    uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + 2 * NS + 6);
    uint32_t* count = reinterpret_cast<uint32_t*>(bars + 2 * NS + 7);      // stages that this CTA asked for
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
        *count = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        for (int i = 0; i < 2; ++i) {
            tma_prefetch(&P.q[i].ma[0][0]);
            tma_prefetch(&P.q[i].mb[0][0]);
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
    stream_order();

    constexpr int kPairs = pairs_of(kParts);      // products of parts per product
    const int unit = blockIdx.x / CG;
    int which;
    long long t;
    // a role that gives up tells the others, in both CTAs
    auto give_up = [&]() {
        *gave_up = 1;
        if (CG == 2)
            asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"(at_cta(smem_u32((const void*)gave_up), rank ^ 1)), "r"(1)
                         : "memory");
        *static_cast<volatile unsigned*>(P.err) = 1u;       // (of the host)
        __threadfence_system();
    };

    // Whole warps walk the loops of the two issuing roles (uniform control flow is cheaper
    // than one lane's); one elected lane issues.
    const bool issuer = elect_one();
    int s = 0;                   // the issuing roles' next stage, its phase
    uint32_t ph = 0;
    bool issued = false;         // products
    if (warp == 0) {
        const uint32_t full0 = CG == 2 ? at_cta(full, 0) : full;
        uint32_t asked = 0;
        bool ok = true;
        for (int i = 0; ok && tile_of(P.plan, unit, i, which, t); ++i) {
            const Problem<kParts>& A = P.q[which];
            const TileAt T = tile_at(A, t);
            const int kblocks = A.kblocks * kPairs * (A.form == SUM ? 2 : 1);
            const int kb0 = (int)((long long)kblocks * T.split / A.splits), kb1 = (int)((long long)kblocks * (T.split + 1) / A.splits);
            const int m0 = T.m * BM * CG + (int)rank * BM;
            const int n0 = T.n * (kGated ? BN / 2 : BN) + (kGated ? 0 : (int)rank * (BN / CG));
            const int depth = A.kblocks * BK;
            // slices of stages, the operands' layouts known
            auto slices = [&](auto a_mn, auto b_mn) {
                int term = kb0 / A.kblocks, k0 = (kb0 - term * A.kblocks) * BK;
                const CUtensorMap *ma, *mb, *mb1;
                auto maps = [&]() {
                    const int sum = term >= kPairs ? 1 : 0, pair = term - sum * kPairs;
                    const int pa = kParts == 3 ? kOrderA >> (2 * pair) & 3 : kParts == 2 ? 1 - pair : 0;
                    const int pb = kParts == 3 ? kOrderB >> (2 * pair) & 3 : 0;
                    ma = &A.ma[T.which + sum][pa];
                    mb = &A.mb[kGated ? (int)rank : T.which + sum][pb];
                    mb1 = &A.mb[1][pb];
                };
                maps();
                for (int kb = kb0; kb < kb1; ++kb, k0 += BK) {
                    if (k0 >= depth) {
                        ++term;
                        k0 = 0;
                        maps();
                    }
                    if (!mbar_wait(empty + 8 * s, ph ^ 1, P.wait_ns, gave_up)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = base + s * S::kStage, sb = sa + kStageA, bar = full0 + 8 * s;
                    if (issuer) {
                        if (rank == 0)
                            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(full + 8 * s),
                                         "r"(CG * S::kStage)
                                         : "memory");
                        if constexpr (decltype(a_mn)::value) {
#pragma unroll
                            for (int j = 0; j < BM / 64; ++j) tma_load<CG>(sa + j * 8192, ma, m0 + 64 * j, k0, bar);
                        } else {
                            tma_load<CG>(sa, ma, k0, m0, bar);
                        }
                        if constexpr (decltype(b_mn)::value) {
#pragma unroll
                            for (int j = 0; j < BN / CG / 64; ++j) tma_load<CG>(sb + j * 8192, mb, n0 + 64 * j, k0, bar);
                        } else {
                            tma_load<CG>(sb, mb, k0, n0, bar);
                            if (kGated && CG == 1) tma_load<CG>(sb + S::kStageB / 2, mb1, k0, n0, bar);
                        }
                    }
                    ++asked;
                    if (++s == NS) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            };
            if constexpr (kGated) {
                slices(Flag<false>{}, Flag<false>{});
            } else {       // forward, gradient of x, gradient of the weight
                if (!A.b_mn) slices(Flag<false>{}, Flag<false>{});
                else if (!A.a_mn) slices(Flag<false>{}, Flag<true>{});
                else slices(Flag<true>{}, Flag<true>{});
            }
        }
        let_next();
        if (issuer) {
            *count = asked;
            if (!ok) give_up();
        }
    } else if (warp == 1 && rank == 0) {
        int acc = 0;
        uint32_t aph = 0;
        bool ok = true;
        for (int i = 0; ok && tile_of(P.plan, unit, i, which, t); ++i) {
            const Problem<kParts>& A = P.q[which];
            const TileAt T = tile_at(A, t);
            const int kblocks = A.kblocks * kPairs * (A.form == SUM ? 2 : 1);
            const int kb0 = (int)((long long)kblocks * T.split / A.splits), kb1 = (int)((long long)kblocks * (T.split + 1) / A.splits);
            const uint32_t idesc = (1u << 4) | ((uint32_t)P.bf16 << 7) | ((uint32_t)P.bf16 << 10) | ((uint32_t)A.a_mn << 15) |
                                   ((uint32_t)A.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM * CG >> 4) << 24);
            const uint32_t step_a = A.a_mn ? 2048 >> 4 : 32 >> 4, step_b = A.b_mn ? 2048 >> 4 : 32 >> 4;
            const int nb = A.kblocks;
            for (int from = kb0; ok && from < kb1;) {      // an accumulator's share: all, or a chunk
                const int end = kSums ? chunk_end<kPairs>(from, kb1, nb) : kb1;
                if (!mbar_wait(tempty + 8 * acc, aph ^ 1, P.wait_ns, gave_up)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                for (int kb = from; kb < end; ++kb) {
                    if (!mbar_wait(full + 8 * s, ph, P.wait_ns, gave_up)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t da = smem_desc(base + s * S::kStage, 8192), db = smem_desc(base + s * S::kStage + kStageA, 8192);
                    if (issuer) {
#pragma unroll
                        for (int j = 0; j < BK / 16; ++j)
                            mma<CG>(tmem + acc * BN, da + j * step_a, db + j * step_b, idesc, kb > from || j > 0);
                        mma_commit<CG>(empty + 8 * s);
                        if (kb + 1 == end) mma_commit<CG>(tfull + 8 * acc);
                    }
                    issued = true;
                    if (++s == NS) {
                        s = 0;
                        ph ^= 1;
                    }
                }
                from = end;
                if (++acc == 2) {
                    acc = 0;
                    aph ^= 1;
                }
            }
        }
        if (!ok && issuer) give_up();
    } else if (warp >= 4) {
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float* stage = staging + (warp - 4) * 2 * 32 * 17;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        constexpr int kCols = kGated ? BN / 2 : BN;   // output columns of a tile
        int acc = 0;
        uint32_t aph = 0;
        for (int i = 0; tile_of(P.plan, unit, i, which, t); ++i) {
            const Problem<kParts>& A = P.q[which];
            const TileAt T = tile_at(A, t);
            if (!A.part) {      // biases of this warp's columns
                __syncwarp();
                for (int w = 0; w < (kGated ? 2 : 1); ++w) {
                    const void* from = A.f.bias[kGated ? w : T.which];
                    if (from)
                        for (int c = lane; c < kCols / 2; c += 32) {
                            const int64_t col = (int64_t)T.n * kCols + half * (kCols / 2) + c;
                            stage[kBias + w * kBiasUp + c] = col < A.f.n ? load_as(from, A.f.dtype, col) : 0.f;
                        }
                }
            }
            const int64_t row0 = ((int64_t)T.m * CG + rank) * BM + quad * 32;
            const int64_t n0 = (int64_t)T.n * kCols;
            auto release = [&]() {       // the accumulator may be written again
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
            };
            if constexpr (!kSums) {
                constexpr int kStep = kCols / 2 < 32 ? 16 : 32;
                const int first = half * (kCols / 2), rows = (int)max((int64_t)0, min((int64_t)32, A.f.m - row0));
                auto whole = [&](int c) { return kStep == 32 && A.vec && !A.part && n0 + c + 32 <= A.f.n; };
                // the residual is asked for one step ahead
                auto ask = [&](int c, uint4 (&r)[4]) {
                    if (!kGated && A.f.res && c < first + kCols / 2 && whole(c))
                        rows_ask(r, static_cast<const char*>(A.f.res) + 2 * (row0 * A.f.ld_res + n0 + c), 2 * A.f.ld_res, rows, lane);
                };
                uint4 res[4] = {}, next[4] = {};
                ask(first, next);
                if (!mbar_wait(tfull + 8 * acc, aph, P.wait_ns, gave_up)) {
                    if (lane == 0) give_up();
                    break;
                }
                tc_fence_after();
#pragma unroll 1
                for (int c = first; c < first + kCols / 2; c += kStep) {
                    const float* bias = stage + kBias + c - first;
#pragma unroll
                    for (int i = 0; i < 4; ++i) res[i] = next[i];
                    ask(c + kStep, next);
                    float v[2][16], u[2][16];
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < kStep / 16; ++h) {
                        tmem_ld(tmem + lanes + acc * BN + c + 16 * h, v[h]);
                        if (kGated) tmem_ld(tmem + lanes + acc * BN + BN / 2 + c + 16 * h, u[h]);
                    }
                    tmem_wait();
                    if (whole(c)) {
                        write32<kGated, kParts>(A, T, row0, n0 + c, lane, v, u, res, bias, stage);
                    } else {
#pragma unroll
                        for (int h = 0; h < kStep / 16; ++h) write16<kGated, kParts, kSums>(A, T, row0, n0 + c + 16 * h, lane, v[h], u[h], bias + 16 * h, stage);
                    }
                }
                release();
            } else {
                constexpr int kSteps = kCols / 32;       // steps of 16 columns
                float v[kSteps][16], u[kSteps][16];
#pragma unroll
                for (int q = 0; q < kSteps; ++q)
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[q][e] = u[q][e] = 0.f;
                const int kblocks = A.kblocks * kPairs * (A.form == SUM ? 2 : 1), nb = A.kblocks;
                const int kb0 = (int)((long long)kblocks * T.split / A.splits), kb1 = (int)((long long)kblocks * (T.split + 1) / A.splits);
                bool ok = true;
                for (int from = kb0; from < kb1; from = chunk_end<kPairs>(from, kb1, nb)) {
                    if (!mbar_wait(tfull + 8 * acc, aph, P.wait_ns, gave_up)) {
                        if (lane == 0) give_up();
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    __syncwarp();
#pragma unroll
                    for (int q = 0; q < kSteps; ++q) {
                        float x[16];
                        tmem_ld(tmem + lanes + acc * BN + half * (kCols / 2) + 16 * q, x);
                        tmem_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[q][e] += x[e];
                        if constexpr (kGated) {
                            tmem_ld(tmem + lanes + acc * BN + BN / 2 + half * (kCols / 2) + 16 * q, x);
                            tmem_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) u[q][e] += x[e];
                        }
                    }
                    release();
                }
                if (!ok) break;
#pragma unroll
                for (int q = 0; q < kSteps; ++q) {
                    write16<kGated, kParts, kSums>(A, T, row0, n0 + half * (kCols / 2) + 16 * q, lane, v[q], u[q], stage + kBias + 16 * q, stage);
                }
            }
        }
    }
    auto meet = [&]() {
        __syncwarp();
        tc_fence_before();
        __syncthreads();
        if (CG == 2) {   // no CTA leaves while its partner may still signal it or read its memory
            asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        }
        tc_fence_after();
    };
    meet();
    if (*gave_up) {      // the same in both CTAs
        if (warp == 1 && issued) {      // products in flight, of any role's giving up
            if (issuer) mma_commit<CG>(drain);
            mbar_wait(drain, 0, kWaitNs, nullptr);
        }
        // Copies in flight, of both CTAs, at the first one's barriers.  A pair's CTAs may have asked for
        // a different number of stages (by NS at most: further ones wait for the products of both
        // halves).  Stage j, counted from the first CTA's next one, is the last use of its place in
        // the ring for each of the NS values of j.
        if (warp == 0 && rank == 0) {
            const uint32_t mine = *count;
            const int ahead = CG == 2 ? (int)(peer_word(smem_u32(count), 1) - mine) : 0, last = max(ahead, 0);
            for (int j = last - NS; j < last; ++j) {
                if (j < 0 && mine < (uint32_t)-j) continue;       // never asked for
                const int at = s + j, q = at < 0 ? at + NS : at >= NS ? at - NS : at;
                const uint32_t bar = full + 8 * q;
                if (CG == 2 && lane == 0) {
                    if (j >= 0)              // the second CTA's half alone: its bytes are announced here
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(S::kStage) : "memory");
                    else if (j >= ahead)     // the first CTA's half alone: the other's bytes never come
                        asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(S::kStage) : "memory");
                }
                __syncwarp();
                if (!mbar_wait(bar, at == q ? ph : ph ^ 1, kWaitNs, nullptr)) break;
            }
        }
        meet();
    }
    if (warp == 2) {
        if (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(S::kTmem) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(S::kTmem) : "memory");
    }
}

// Nanoseconds after which a wait gives up: VQC_WAIT_NS of the environment, or 4 s.
unsigned long long wait_limit() {
    static const unsigned long long ns = [] {
        const char* v = std::getenv("VQC_WAIT_NS");
        const unsigned long long given = v ? std::strtoull(v, nullptr, 10) : 0;
        return given ? given : kWaitNs;
    }();
    return ns;
}

// A word per device that a kernel sets when it gave up, in memory of the host, where every later call
// looks at it for nothing.
constexpr int kDevices = 64;
std::atomic<unsigned*> g_words{nullptr};

cudaError_t error_word(unsigned** p) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= kDevices) return cudaErrorInvalidDevice;
    unsigned* words = g_words.load();
    if (!words) {
        static std::mutex mu;
        std::lock_guard<std::mutex> lk(mu);
        words = g_words.load();
        if (!words) {
            // (allowed while a stream is captured: nothing of it enters the graph)
            cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
            cudaThreadExchangeStreamCaptureMode(&mode);
            void* q = nullptr;
            e = cudaHostAlloc(&q, kDevices * sizeof(unsigned), cudaHostAllocPortable | cudaHostAllocMapped);
            cudaThreadExchangeStreamCaptureMode(&mode);
            if (e != cudaSuccess) return e;
            words = static_cast<unsigned*>(q);
            std::fill(words, words + kDevices, 0u);
            g_words.store(words);
        }
    }
    return cudaHostGetDevicePointer(reinterpret_cast<void**>(p), words + dev, 0);
}
// the current device's word as the host reads it, or NULL where no product has run
volatile unsigned* host_word() {
    unsigned* words = g_words.load();
    int dev = 0;
    return words && cudaGetDevice(&dev) == cudaSuccess && dev < kDevices ? words + dev : nullptr;
}

// A float as the sum of three bf16, 8 bits of it each: exact for normal results.  The six products
// of parts (kOrderA, kOrderB) have to make float's infinities and NaN of two operands' parts:
//   - a value below 2^8 is rounded to nearest at each part, so that what the six products drop has either sign;
//   - above, where a product of two such parts could leave the range with the other sign, it is cut, all
//     parts with its sign (an infinity of the whole product is then that of its parts);
//   - an infinity is 1, 0 and the infinity: that third part meets the other operand's first
//     part only, which is zero, positive or negative as the operand is (1 where that is an infinity too).  A
//     NaN, so placed, is in every sum.
// (A finite product within 2^-8 of the largest float may come out infinite, and a finite operand
// below 2^-134 counts as zero beside an infinite one.)
__device__ __forceinline__ void bf16_parts(float x, uint16_t (&o)[3]) {
    const float size = fabsf(x);
    if (!(size <= 3.4028234e38f)) {
        o[0] = 0x3f80 | (uint16_t)(__float_as_uint(x) >> 16 & 0x8000);
        o[1] = 0;
        o[2] = __bfloat16_as_ushort(__float2bfloat16(x));
        return;
    }
    float rest = x;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const uint16_t near = __bfloat16_as_ushort(__float2bfloat16(rest));
        o[i] = size < 256.f ? near : (uint16_t)(__float_as_uint(rest) >> 16);
        rest -= __uint_as_float((uint32_t)o[i] << 16);
    }
}

// Copies of operands that TMA cannot read in place, up to four in one launch (job
// blockIdx.y): [rows, cols] with rows of `ld_to` elements (a multiple of 8).  Floats
// become three matrices of parts, 16-bit elements keep their bits.  8 elements
// per thread, bound by bytes: 10240 x 1177 bfloat16 10.6 us.
struct CopyJob {
    const void* from;
    uint16_t* to;
    int64_t ld, rows, cols, ld_to;
    int vec;            // rows of `from` on 16-byte boundaries
};
constexpr int kMostCopies = 8;
struct CopyJobs {
    CopyJob j[kMostCopies];
    int count;
};
template <int kParts> __global__ void __launch_bounds__(256) copy_kernel(const __grid_constant__ CopyJobs J) {
    stream_order();
    const CopyJob& A = J.j[blockIdx.y];
    const int64_t across = A.ld_to / 8, plane = A.rows * A.ld_to, count = A.rows * across, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < count; e += step) {
        const int64_t r = count >> 32 ? e / across : (int64_t)((uint32_t)e / (uint32_t)across), c = (e - r * across) * 8;
        uint16_t* to = A.to + r * A.ld_to + c;
        if constexpr (kParts == 1) {
            const uint16_t* p = static_cast<const uint16_t*>(A.from) + r * A.ld + c;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (c + 2 * i < A.cols ? (uint32_t)p[2 * i] : 0u) | (c + 2 * i + 1 < A.cols ? (uint32_t)p[2 * i + 1] << 16 : 0u);
            *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            const float* p = static_cast<const float*>(A.from) + r * A.ld + c;
            float v[8];
            if (A.vec && c + 8 <= A.cols) {
                const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
                v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = c + i < A.cols ? p[i] : 0.f;
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
                *reinterpret_cast<uint4*>(to + q * plane) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
        }
    }
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

// The tile, and the cuts of each of up to two products.
struct Choice {
    int cg, bn, splits[2];
};
struct TileKind {
    int cg, bn;
    double stage;      // cycles of one stage of 64
};
constexpr TileKind kTiles[] = {{2, 256, 560}, {2, 128, 400}, {1, 128, 512}, {1, 64, 384}};

int64_t tiles_of(const Product& p, const TileKind& t) {
    return ceil_div(p.m, BM * t.cg) * ceil_div(p.n, p.form == GATED ? t.bn / 2 : t.bn) * (p.form == PAIR ? 2 : 1);
}
int parts_in(const Product& p) { return p.f.dtype == VQC_F32 ? 3 : p.a[0].second ? 2 : 1; }
int64_t depth_of(const Product& p) { return ceil_div(p.k, BK) * (p.form == SUM ? 2 : 1) * pairs_of(parts_in(p)); }

// The schedule of `first` tiles of c0 cycles and `second` of c1 <= c0, and its length.
double make_schedule(int64_t first, double c0, int64_t second, double c1, int units, Schedule& s) {
    s.first = first;
    s.second = second;
    s.units = (int)std::min<int64_t>(units, first + second);
    s.rounds = (int)(first / s.units);
    s.extra = (int)(first % s.units);
    s.second_rounds = 0;
    const double most = (s.rounds + (s.extra ? 1 : 0)) * c0;
    if (!second) return most;
    if (!s.extra) {
        s.second_rounds = (int)ceil_div(second, s.units);
        return most + s.second_rounds * c1;
    }
    const int rest = s.units - s.extra;
    const int64_t guess = (int64_t)(((first * c0 + second * c1) / s.units - most) / c1);
    double best = 1e300;
    for (int64_t r = std::max<int64_t>(0, guess - 1); r <= std::max<int64_t>(0, guess) + 1; ++r) {
        const int64_t left = std::max<int64_t>(0, second - r * s.units);
        const double span = std::max(most + std::min<int64_t>(r, ceil_div(second, s.units)) * c1, s.rounds * c0 + (r + ceil_div(left, rest)) * c1);
        if (span < best) {
            best = span;
            s.second_rounds = (int)r;
        }
    }
    return best;
}

// Taking out an accumulator: measured about 2500 cycles for 256 columns in whole pieces of
// 16 bytes, five times that where rows are turned element by element.
double end_cycles(const Product& p, const TileKind& t) { return (p.n % 8 == 0 ? 10.0 : 50.0) * t.bn; }
// Cycles of a tile: its stages (the products, 8192 per cycle and SM, or the bytes from the
// L2, whichever takes longer), or taking out its accumulator.
double tile_cycles(const Product& p, const TileKind& t, int64_t splits) {
    return std::max((double)ceil_div(depth_of(p), splits) * t.stage, end_cycles(p, t));
}
// of a cut: sums written and read once by all SMs together (and 5000 for the launch of the
// join); 256 x 4096 x 4096 takes 17.4 us in tiles of 256 x 128 and 23.6 cut in two in 128 x 128
double cut_cycles(const Product& p, int64_t splits, int sms) {
    return splits > 1 ? (double)(splits + 1) * p.m * p.n * (p.form == GATED || p.form == PAIR ? 2 : 1) * 4 / (sms * 12.0) : 0.0;
}

// The first of two products is the one with the longer tiles.
bool swapped(const Product* p, int count, const TileKind& t, const int* splits) {
    return count == 2 && tile_cycles(p[0], t, splits[0]) < tile_cycles(p[1], t, splits[1]);
}
double schedule_of(const Product* p, int count, const TileKind& t, const int* splits, int sms, Schedule& s) {
    const int a = swapped(p, count, t, splits), b = 1 - a;
    return make_schedule(tiles_of(p[a], t) * splits[a], tile_cycles(p[a], t, splits[a]), count == 2 ? tiles_of(p[b], t) * splits[b] : 0,
                         count == 2 ? tile_cycles(p[b], t, splits[b]) : 1.0, sms / t.cg, s);
}

// float32 outputs (and operands): sums of chunks in the epilogue's registers, tiles up to 128 columns.
// (The two products of a backward have one type of output.)
bool in_chunks(const Product& p) { return p.f.out_dtype == VQC_F32 || p.f.dtype == VQC_F32; }

Choice choose_new(const Product* p, int count, int sms) {
    static constexpr int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    Choice best{1, 64, {1, 1}};
    double least = 1e300;
    for (const TileKind& t : kTiles) {
        if (in_chunks(p[0]) && t.bn == 256) continue;
        for (int s0 : kCuts) {
            if (s0 > depth_of(p[0])) break;
            for (int s1 : kCuts) {
                if (s1 > (count == 2 ? depth_of(p[1]) : 1)) break;
                const int splits[2] = {s0, s1};
                Schedule plan;
                double c = schedule_of(p, count, t, splits, sms, plan) + end_cycles(p[0], t) + cut_cycles(p[0], s0, sms);
                if (count == 2) c += cut_cycles(p[1], s1, sms);
                if (s0 > 1 || s1 > 1) c += 5000;
                if (c < least) {
                    least = c;
                    best = {t.cg, t.bn, {s0, s1}};
                }
            }
        }
    }
    return best;
}

// The choices of the sizes that a thread asked for last.
Choice choose(const Product* p, int count) {
    struct Key {
        int64_t v[9];
        bool operator==(const Key& o) const { return std::equal(v, v + 9, o.v); }
    };
    struct Known {
        Key key{};
        Choice c{};
    };
    static thread_local Known known[64];
    const int sms = sm_count();
    Key key{};
    uint64_t hash = 0;
    key.v[0] = sms;
    for (int i = 0; i < count; ++i) {
        key.v[4 * i + 1] = p[i].m; key.v[4 * i + 2] = p[i].n; key.v[4 * i + 3] = p[i].k;
        key.v[4 * i + 4] = 1 + p[i].form + 8 * parts_in(p[i]) + 64 * in_chunks(p[i]);
    }
    for (int64_t v : key.v) hash = (hash ^ (uint64_t)v) * 0x9E3779B97F4A7C15ull;
    Known& q = known[hash >> 58];
    if (!(q.key == key)) {
        q.c = choose_new(p, count, sms);
        q.key = key;
    }
    return q.c;
}

template <int CG, int BN, bool kGated, int kParts, bool kSums> cudaError_t launch_tc(const TcArgs<kParts>& a, cudaStream_t s) {
    using S = Shape<CG, BN>;
    void* args[] = {const_cast<TcArgs<kParts>*>(&a)};
    return launch((const void*)tc_kernel<CG, BN, kGated, kParts, kSums>, dim3((unsigned)(a.plan.units * CG)), kThreads, args, s, S::kSmem, CG);
}

template <bool kGated, int kParts, bool kSums> cudaError_t launch_choice(const Choice& c, const TcArgs<kParts>& a, cudaStream_t s) {
    if constexpr (!kSums)
        if (c.cg == 2 && c.bn == 256) return launch_tc<2, 256, kGated, kParts, false>(a, s);
    if (c.cg == 2) return launch_tc<2, 128, kGated, kParts, kSums>(a, s);
    return c.bn == 128 ? launch_tc<1, 128, kGated, kParts, kSums>(a, s) : launch_tc<1, 64, kGated, kParts, kSums>(a, s);
}

int left_operands(const Product& p) { return p.form == SUM || p.form == PAIR ? 2 : 1; }
int right_operands(const Product& p) { return p.form == SUM || p.form == GATED ? 2 : 1; }

size_t space(const Product& p, bool aligned, int splits) {
    size_t bytes = 0;
    for (int i = 0; i < left_operands(p); ++i)
        if (!ready(p.a[i], p.f.dtype, aligned)) bytes += copy_bytes(p.a[i], p.f.dtype, p.m, p.k);
    for (int i = 0; i < right_operands(p); ++i)
        if (!ready(p.b[i], p.f.dtype, aligned)) bytes += copy_bytes(p.b[i], p.f.dtype, p.n, p.k);
    if (splits > 1) bytes += align256((size_t)splits * (p.form == GATED || p.form == PAIR ? 2 : 1) * p.m * p.n * 4);
    return bytes;
}

// The copies that a product's operands need (one copy of a matrix that two products
// read), and the operands as the kernel reads them.
struct Placed {
    Operand a[2], b[2];
    char* at;         // what is left of the workspace
    size_t left;
};
vqc_status place(const Product& p, void* ws, size_t ws_bytes, CopyJobs& jobs, Placed& r) {
    r.at = static_cast<char*>(ws);
    r.left = ws ? ws_bytes : 0;
    for (int side = 0; side < 2; ++side)
        for (int i = 0; i < (side ? right_operands(p) : left_operands(p)); ++i) {
            Operand o = side ? p.b[i] : p.a[i];
            const int64_t outer = side ? p.n : p.m;
            if (!ready(o, p.f.dtype, aligned_to(o.p, 16))) {
                CopyJob j{o.p, nullptr, o.ld, o.k_outer ? p.k : outer, o.k_outer ? outer : p.k, 0, o.ld % 4 == 0 && aligned_to(o.p, 16)};
                j.ld_to = copy_ld(j.cols);
                const CopyJob* same = nullptr;
                for (int q = 0; q < jobs.count; ++q)
                    if (jobs.j[q].from == j.from && jobs.j[q].ld == j.ld && jobs.j[q].rows == j.rows && jobs.j[q].cols == j.cols) same = &jobs.j[q];
                if (!same) {
                    const size_t bytes = copy_bytes(o, p.f.dtype, outer, p.k);
                    if (bytes > r.left || jobs.count == kMostCopies) return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
                    j.to = reinterpret_cast<uint16_t*>(r.at);
                    r.at += bytes;
                    r.left -= bytes;
                    same = &(jobs.j[jobs.count++] = j);
                }
                o.p = same->to;
                o.ld = same->ld_to;
            }
            (side ? r.b : r.a)[i] = o;
        }
    return VQC_OK;
}

template <int kParts> vqc_status fill_problem(const Product& p, const Choice& c, int splits, Placed& r, Problem<kParts>& a, Joins& joins) {
    const bool gated = p.form == GATED;
    const int na = left_operands(p), nb = right_operands(p);
    for (int side = 0; side < 2; ++side)
        for (int i = 0; i < (side ? nb : na); ++i) {
            const Operand& o = (side ? r.b : r.a)[i];
            const int64_t outer = side ? p.n : p.m, rows = o.k_outer ? p.k : outer;
            const int box = side ? (gated ? c.bn / 2 : c.bn / c.cg) : BM;
            for (int q = 0; q < (side ? Problem<kParts>::kPartsB : kParts); ++q) {
                Operand part = o;
                part.p = static_cast<const uint16_t*>(o.p) + q * (kParts == 2 ? o.second : rows * o.ld);
                if (!make_map(side ? &a.mb[i][q] : &a.ma[i][q], part, p.f.dtype, outer, p.k, box))
                    return set_error(VQC_ERR_CUDA, "product: cuTensorMapEncodeTiled failed");
            }
        }
    // an operand of both products
    for (int q = 0; q < kParts && na == 1; ++q) a.ma[1][q] = a.ma[0][q];
    for (int q = 0; q < Problem<kParts>::kPartsB && nb == 1; ++q) a.mb[1][q] = a.mb[0][q];
    if (splits < 1 || splits > depth_of(p)) return set_error(VQC_ERR_DEVICE_CHECK, "product: more cuts than blocks");   // a tile with nothing to add
    a.f = p.f;
    a.form = p.form;
    a.splits = splits;
    a.tiles_m = (int)ceil_div(p.m, BM * c.cg);
    a.tiles_n = (int)ceil_div(p.n, gated ? c.bn / 2 : c.bn);
    a.kblocks = (int)ceil_div(p.k, BK);
    a.a_mn = p.a[0].k_outer;
    a.b_mn = p.b[0].k_outer;
    a.part = nullptr;
    if (splits > 1) {
        if (align256((size_t)splits * (gated || p.form == PAIR ? 2 : 1) * p.m * p.n * 4) > r.left)
            return set_error(VQC_ERR_WORKSPACE, "product: workspace too small");
        a.part = reinterpret_cast<float*>(r.at);
        Join& j = joins.j[joins.count++];
        j.f = p.f;
        j.part = a.part;
        j.splits = splits;
        j.form = p.form;
    }
    // the widest store that every row of every output allows
    const int64_t eo = (int64_t)elem_size(p.f.out_dtype);
    auto on = [&](int w) {
        if (a.part) return p.n * 4 % w == 0;
        return p.n * eo % w == 0 && aligned_to(p.f.y[0], w) && aligned_to(p.f.y[1], w) &&
               (!p.f.z[0] || (p.n * 4 % w == 0 && aligned_to(p.f.z[0], w) && aligned_to(p.f.z[1], w))) &&
               (!p.f.res || (p.f.ld_res * eo % w == 0 && aligned_to(p.f.res, w)));
    };
    a.vec = on(32) ? 32 : on(16) ? 16 : 0;
    return VQC_OK;
}

template <int kParts> vqc_status run_parts(const Product* p, int count, void* const* ws, const size_t* bytes, Joins& joins, cudaStream_t s) {
    const Choice c = choose(p, count);
    const bool gated = p[0].form == GATED;
    CopyJobs jobs;
    jobs.count = 0;
    Placed placed[2];
    for (int i = 0; i < count; ++i) {
        const vqc_status st = place(p[i], ws[i], bytes[i], jobs, placed[i]);
        if (st != VQC_OK) return st;
    }
    if (jobs.count) {
        int64_t most = 1;
        for (int i = 0; i < jobs.count; ++i) most = std::max(most, jobs.j[i].rows * jobs.j[i].ld_to / 8);
        void* args[] = {&jobs};
        const cudaError_t e = launch((const void*)copy_kernel<kParts == 3 ? 3 : 1>, dim3((unsigned)std::min<int64_t>(ceil_div(most, 256), 8LL * sm_count()), jobs.count), 256, args, s);
        if (e != cudaSuccess) return cuda_error(e, "operand copy launch");
    }
    const TileKind* tile = kTiles;
    while (tile->cg != c.cg || tile->bn != c.bn) ++tile;
    TcArgs<kParts> a;
    schedule_of(p, count, *tile, c.splits, sm_count(), a.plan);
    const int order = swapped(p, count, *tile, c.splits);
    for (int i = 0; i < count; ++i) {
        const int from = order ? 1 - i : i;
        const vqc_status st = fill_problem<kParts>(p[from], c, c.splits[from], placed[from], a.q[i], joins);
        if (st != VQC_OK) return st;
    }
    if (count == 1) a.q[1] = a.q[0];
    a.bf16 = p[0].f.dtype != VQC_F16;
    a.wait_ns = wait_limit();
    cudaError_t e = error_word(&a.err);
    if (e != cudaSuccess) return cuda_error(e, "cudaGetSymbolAddress");
    if constexpr (kParts == 3) {
        e = gated ? launch_choice<true, 3, true>(c, a, s) : launch_choice<false, 3, true>(c, a, s);
    } else if constexpr (kParts == 2) {
        e = launch_choice<false, 2, false>(c, a, s);
    } else {
        e = gated             ? launch_choice<true, 1, false>(c, a, s)
            : in_chunks(p[0]) ? launch_choice<false, 1, true>(c, a, s)
                              : launch_choice<false, 1, false>(c, a, s);
    }
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "tensor-core product launch");
}

}  // namespace

// 16-bit products with anything to add up, and float products where six products of parts
// (and writing the parts) take less time than float FMAs: 1000^3 35 us against 195 on the FP32
// units, 512 x 512 x 512 about 19 either way.
bool tc_takes(const Product& p) {
    if (p.m <= 0 || p.k <= 0) return false;
    if (p.f.dtype != VQC_F32) return true;
    const double flops = 2.0 * p.m * p.n * p.k * (p.form == PLAIN ? 1 : 2);
    return flops >= 5e8 && p.k >= 64 && std::min(p.m, p.n) >= 64;
}

void tc_workspace(const Product* p, int count, bool aligned, size_t* bytes) {
    const Choice both = choose(p, count);
    for (int i = 0; i < count; ++i) {
        bytes[i] = space(p[i], aligned, both.splits[i]);
        if (count == 2) bytes[i] = std::max(bytes[i], space(p[i], aligned, choose(p + i, 1).splits[0]));   // either may run alone
    }
}

vqc_status tc_run(const Product* p, int count, void* const* ws, const size_t* bytes, Joins& joins, cudaStream_t s) {
    switch (parts_in(p[0])) {
        case 3: return run_parts<3>(p, count, ws, bytes, joins, s);
        case 2: return run_parts<2>(p, count, ws, bytes, joins, s);
        default: return run_parts<1>(p, count, ws, bytes, joins, s);
    }
}

}  // namespace layers

// What an earlier product's wait left behind: reported to every call until vqc_sync_check has been told.
vqc_status layers_pending() {
    const volatile unsigned* w = layers::host_word();
    if (!w || !*w) return VQC_OK;
    return set_error(VQC_ERR_DEVICE_CHECK, "an earlier tensor-core product's wait timed out and its output is incomplete (vqc_sync_check "
                                           "reports this and clears it)");
}

// vqc_sync_check's view of the error word (read and cleared).
vqc_status layers_error_check() {
    volatile unsigned* w = layers::host_word();
    if (!w || !*w) return VQC_OK;
    *w = 0;
    return set_error(VQC_ERR_DEVICE_CHECK, "a tensor-core product's wait timed out");
}

}  // namespace vqc
