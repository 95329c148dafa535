// attention_tc.cu -- attention on the tensor cores (tcgen05) for 16-bit types and heads of up to 128
// elements; the formulas are those of attention.cu.
//
// Forward.  A CTA owns 256 queries of a head, two halves of 128 rows, and goes through the tiles of 128 keys that
// one of them sees.  Warp 0 moves tiles of keys and values into a ring with TMA, warp 1 issues the products:
// scores S = Q K^T into tensor memory, and O += P V with P read from tensor memory (it lies where S lay).
// Warps 4..7 and 8..11 take the scores of one half out, a row per lane, and put the probabilities back: while one half's are
// worked on, the tensor cores multiply the other's.  A row's running maximum is followed only when it has grown by
// more than 2^8: P and the row's sum are relative to the followed one, and O is rescaled in tensor memory
// then (the product that last wrote it has ended: its scores' successor was committed after it).
//
// 4 x 4096 tokens, 16 heads over 4 of 128 elements, bfloat16: 176 us, 1560 TFLOP/s of visible pairs (16384 tokens: 610 us, 1800).
// Bound by the products: a 128 x 128 x 16 one takes 64 cycles with its left operand in tensor memory (P V) and about 100
// with both in shared memory (Q K^T).
//
// P is rounded to the operands' type (one rounding of a probability, whose error averages out over the keys
// of a row), its sum is taken before.  float16 probabilities are held times 2^6: 2^-30 of the largest.
//
// Every wait is bounded, as in layers_tc.cu: a warp that gives up tells the others, copies and products
// in flight are waited for, tensor memory is freed and the error word set.
#include <algorithm>
#include <type_traits>

#include "attention.h"
#include "layers_elem.cuh"
#include "layers_tc.h"
#include "tensor_core.cuh"

namespace vqc {
namespace layers {

namespace {

constexpr int N = 128;                               // queries of a half, keys of a tile
constexpr int kThreads = 384;
constexpr int kChunk = N * 128;                      // 128 rows of 64 elements, 128-byte swizzle
constexpr int kBarriers = 1024;
constexpr unsigned long long kWaitNs = 4000000000ull;   // bound of the waits for what is in flight
constexpr float kLn2 = 0.693147180559945309f;

// Which keys a query sees, in 32 bits (tokens are below 2^30; so are a window and sinks that matter).
struct View {
    const int32_t* lengths;
    int tokens, window, sinks;
    __device__ __forceinline__ int length(int b) const { return lengths ? min(max(lengths[b], 0), tokens) : tokens; }
};

struct TcAttention {
    CUtensorMap q, k, v, g;
    View sight;
    void* o;
    float* saved;
    unsigned* err;
    unsigned long long wait_ns;
    int tiles, items;            // tiles of a head, of all heads of all sequences
    float scale, scale2;
    int heads, groups, dim;
};

// The tiles of keys that rows first..last - 1 see: [0, sinks) and [from, to); none where there are no rows.
struct Span {
    int sinks, from, to;
    __device__ __forceinline__ bool has(int t) const { return t < sinks || (t >= from && t < to); }
};
__device__ __forceinline__ Span span_of(const View& S, int first, int last) {
    Span r{0, 0, 0};
    if (first >= last) return r;
    r.to = (last + N - 1) / N;
    r.from = max(0, first - S.window + 1) / N;
    r.sinks = min((min(S.sinks, S.tokens) + N - 1) / N, r.from);
    return r;
}
// All keys of a tile are seen by all rows first..first + N - 1 (of those that there are)?
__device__ __forceinline__ bool all_seen(const View& S, int first, int tile) {
    const int k0 = tile * N, k1 = k0 + N - 1;
    return k1 <= first && (first + N - 1 - k0 < S.window || k1 < S.sinks);
}

// 2^x, zero below the smallest normal number (without that, three more instructions)
__device__ __forceinline__ float power(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the n lowest bits (none below 0, all from 32 on)
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// The end of a wait that was not over at the first look, out of line: in the place of every wait its code made a unit of the
// backward last 900 cycles even without products and arithmetic, for instructions to be fetched (640 so), and a
// forward of 4 x 4096 tokens, 16 heads, 208 us (194).
static __device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, unsigned long long ns, const volatile int* gave_up) {
    // (a bound of milliseconds is looked at after some tries, each of which waits by itself: reading the clock takes long)
    const int tries = ns >= 1000000 ? 32 : 0;
#pragma unroll 1
    for (int i = 0; i < tries; ++i)
        if (__all_sync(~0u, mbar_try(bar, parity))) return true;
    const unsigned long long end = now_ns() + ns;
    for (;;) {
        if (__all_sync(~0u, mbar_test(bar, parity))) return true;
        if (__any_sync(~0u, *gave_up || now_ns() > end)) return false;
    }
}
// The pieces that every kernel here has: barriers, a bounded end.
struct Roles {
    const volatile int* gave_up;
    unsigned long long ns;
    // False when the bound ran out or another role gave up.  The first look waits by itself, for a time that the device bounds.
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
        return __all_sync(~0u, mbar_try(bar, parity)) || __any_sync(~0u, wait_on(bar, parity, ns, gave_up));
    }
    // The same for a free stage, whose warp is ahead of the others and can afford to keep bounds below a millisecond as well
    // (the choice in every wait took 3% of the forward).
    __device__ __forceinline__ bool wait_free(uint32_t bar, uint32_t parity) const {
        return __all_sync(~0u, mbar_look(bar, parity, ns >= 1000000)) || __any_sync(~0u, wait_on(bar, parity, ns, gave_up));
    }
};
__device__ __forceinline__ void give_up(volatile int* flag, unsigned* err) {
    *flag = 1;
    *static_cast<volatile unsigned*>(err) = 1u;       // (of the host)
    __threadfence_system();
}
// A ring of stages, counted.
template <int NS> struct Ring {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++slot == NS) {
            slot = 0;
            phase ^= 1;
        }
    }
};

// zeros in the rows of a tile from `row` on (its chunks of `rows` rows lie one after the other), by one warp
__device__ __forceinline__ void clear_rows(unsigned char* tile, int chunks, int rows, int row, int lane) {
    for (int c = 0; c < chunks; ++c)
        for (int i = row * 8 + lane; i < rows * 8; i += 32) *reinterpret_cast<uint4*>(tile + c * rows * 128 + i * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    __syncwarp();
}

// A warp's 32 rows x 64 elements (a row per lane, packed) to memory by way of shared memory, so that eight lanes
// write 128 bytes of a row: straight from the lanes a store touches 32 lines, 4100 cycles for a CTA's output.
// Piece c (16 bytes) of row r lies at place c ^ (r % 8).  `rows`: rows that exist; `cols`: elements that exist.
__device__ __forceinline__ void rows_out(unsigned char* stage, const uint32_t (&w)[32], char* to, int64_t pitch, int rows, int cols, int lane) {
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c)
        *reinterpret_cast<uint4*>(stage + lane * 128 + ((c ^ (lane & 7)) << 4)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    __syncwarp();
    const int c = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        if (r < rows && 8 * c < cols)
            *reinterpret_cast<uint4*>(to + r * pitch + 16 * c) = *reinterpret_cast<const uint4*>(stage + r * 128 + ((c ^ (r & 7)) << 4));
    }
}

// C chunks of 64 elements in a head.  Stage i of the ring holds the values of tile i - 1 and the keys of
// tile i, which are used one after the other.
template <int C> struct ForwardShape {
    static constexpr int kTile = C * kChunk;
    static constexpr int kStages = C == 1 ? 4 : 2;
    static constexpr int kOut = (2 + 2 * kStages) * kTile;      // where the warps' outputs are turned
    static constexpr int kSmem = kOut + 8 * 4096 + kBarriers;
};

// 256 queries of a head of a sequence.
struct Place {
    int b, head, q0, length;
};
// The n-th of a CTA: long ones first, and every second round of CTAs in the other order.
__device__ __forceinline__ bool place_of(const TcAttention& A, int n, int rows, Place& w) {
    const int64_t i = (int64_t)n * gridDim.x + (n & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    if (i >= A.items) return false;
    const int plane = A.items / A.tiles, tile = A.tiles - 1 - (int)i / plane, which = (int)i % plane;
    w.b = which / A.heads;
    w.head = which - w.b * A.heads;
    w.length = __shfl_sync(~0u, A.sight.length(w.b), 0);
    w.q0 = tile * rows;
    return true;
}
// The tiles that one of its halves sees: [0, sinks) and [from, to).
struct Item : Place {
    int group, sinks, from, count;
    Span half[2];
    __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : from + i - sinks; }
};
__device__ __forceinline__ bool item_of(const TcAttention& A, int n, Item& w) {
    if (!place_of(A, n, 2 * N, w)) return false;
    w.group = w.head / (A.heads / A.groups);
    for (int h = 0; h < 2; ++h) w.half[h] = span_of(A.sight, w.q0 + h * N, min(w.q0 + (h + 1) * N, w.length));
    const int to = max(w.half[0].to, w.half[1].to);
    w.from = w.half[0].from;
    w.sinks = min(max(w.half[0].sinks, w.half[1].sinks), w.from);
    w.count = to ? w.sinks + to - w.from : 0;
    return true;
}

template <typename T, int C> __global__ void __launch_bounds__(kThreads, 1) forward_tc(const __grid_constant__ TcAttention A) {
    using L = ForwardShape<C>;
    constexpr int NS = L::kStages;
    constexpr float kShift = std::is_same<T, __nv_bfloat16>::value ? 0.f : 6.f, kGrowth = 8.f;
    extern __shared__ __align__(1024) unsigned char sm[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + L::kOut + 8 * 4096);
    const uint32_t full = smem_u32(bars), empty = full + 8 * NS, qfull = empty + 8 * NS, qempty = qfull + 16, sfull = qempty + 16, ready = sfull + 16,
                   ofull = ready + 32, drain = ofull + 16;
    volatile int* gave_up = reinterpret_cast<volatile int*>(bars + 2 * NS + 14);
    uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + 2 * NS + 15);
    // (by a shuffle the compiler knows that a warp's role and what follows from it are the same in all lanes, so that the products'
    // operands are in uniform registers: 194 to 180 us with the constant address of tensor memory)
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = smem_u32(sm), ring = base + 2 * L::kTile;

    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int h = 0; h < 2; ++h) {
            mbar_init(qfull + 8 * h, 1);
            mbar_init(qempty + 8 * h, 1);
            mbar_init(sfull + 8 * h, 1);
            mbar_init(ready + 16 * h, 4);
            mbar_init(ready + 16 * h + 8, 4);
            mbar_init(ofull + 8 * h, 1);
        }
        mbar_init(drain, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        tma_prefetch(&A.q);
        tma_prefetch(&A.k);
        tma_prefetch(&A.v);
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tslot)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr uint32_t tmem = 0;      // (all 512 columns are this CTA's)
    stream_order();

    const Roles R{gave_up, A.wait_ns};
    const bool issuer = elect_one();
    uint32_t asked = 0, queries[2] = {0, 0};      // stages and halves asked for
    bool issued = false;
    if (warp == 0) {
        Ring<NS> r;
        Item w;
        bool ok = true;
        for (int n = 0; ok && item_of(A, n, w); ++n) {
            if (!w.count) continue;
            for (int h = 0; ok && h < 2; ++h) {
                if (!w.half[h].to) continue;
                ok = R.wait_free(qempty + 8 * h, (queries[h] & 1) ^ 1);
                if (!ok) break;
                if (issuer) {
                    mbar_expect(qfull + 8 * h, L::kTile);
                    for (int c = 0; c < C; ++c)
                        tma_load4(base + h * L::kTile + c * kChunk, &A.q, 64 * c, w.q0 + h * N, w.head, w.b, qfull + 8 * h);
                }
                ++queries[h];
            }
            for (int i = 0; ok && i <= w.count; ++i) {
                ok = R.wait_free(empty + 8 * r.slot, r.phase ^ 1);
                if (!ok) break;
                if (issuer) {
                    const uint32_t values = ring + r.slot * 2 * L::kTile, bar = full + 8 * r.slot;
                    mbar_expect(bar, (i > 0 && i < w.count ? 2 : 1) * L::kTile);
                    if (i < w.count)
                        for (int c = 0; c < C; ++c) tma_load4(values + L::kTile + c * kChunk, &A.k, 64 * c, w.tile(i) * N, w.group, w.b, bar);
                    if (i > 0)
                        for (int c = 0; c < C; ++c) tma_load4(values + c * kChunk, &A.v, 64 * c, w.tile(i - 1) * N, w.group, w.b, bar);
                }
                ++asked;
                r.next();
            }
        }
        let_next();
        if (!ok && issuer) give_up(gave_up, A.err);
    } else if (warp == 1) {
        // Strictly one half after the other: while one's scores are worked on, the other's are multiplied.  One thread
        // issues all products: products are ordered among those that one thread issues.  (A version with a warp per half, whose last
        // commits nobody waited for, gave wrong outputs; which of the two was its fault was not found.)
        constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u << 7 | 1u << 10 : 0u;
        const uint32_t scores = 1u << 4 | kType | (uint32_t)(N >> 3) << 17 | (uint32_t)(N >> 4) << 24;
        const uint32_t outputs = 1u << 4 | kType | 1u << 16 | (uint32_t)(64 * C >> 3) << 17 | (uint32_t)(N >> 4) << 24;
        Ring<NS> r;
        uint32_t taken[2] = {0, 0};
        Item w;
        bool ok = true;
        for (int n = 0; ok && item_of(A, n, w); ++n) {
            if (!w.count) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!w.half[h].to) continue;
                ok = ok && R.wait(qfull + 8 * h, queries[h] & 1);
                ++queries[h];
            }
            const int tail = w.length < A.sight.tokens ? w.length % N : 0;      // rows behind the sequence: values there are not read
            bool before[2] = {false, false}, any[2] = {false, false};      // the last tile was of this half, a tile was
            for (int i = 0; ok && i <= w.count; ++i) {
                ok = R.wait(full + 8 * r.slot, r.phase);
                if (!ok) break;
                tc_fence_after();
                const uint32_t values = ring + r.slot * 2 * L::kTile;
                const uint64_t dv = smem_desc(values, kChunk), dk = smem_desc(values + L::kTile, 0);
                if (i > 0 && tail && w.tile(i - 1) == w.length / N) clear_rows(sm + (2 + 2 * r.slot) * L::kTile, C, N, tail, lane);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t ts = tmem + h * N, to_o = tmem + 2 * N + h * 64 * C;
                    const bool now = i < w.count && w.half[h].has(w.tile(i));
                    if (before[h]) {
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            ok = ok && R.wait(ready + 16 * h + 8 * part, taken[h] & 1);
                            tc_fence_after();
                            if (issuer && ok) {
#pragma unroll
                                for (int j = part * N / 32; j < (part + 1) * N / 32; ++j) mma_rows(to_o, ts + 8 * j, dv + j * (2048 >> 4), outputs, any[h] || j > 0);
                            }
                        }
                        ++taken[h];
                        any[h] = true;
                    }
                    if (issuer && ok) {
                        if (now) {
                            const uint64_t dq = smem_desc(base + h * L::kTile, 0);
#pragma unroll
                            for (int j = 0; j < 4 * C; ++j) {
                                const uint32_t step = (j / 4 * kChunk + j % 4 * 32) >> 4;
                                mma<1>(ts, dq + step, dk + step, scores, j > 0);
                            }
                            mma_commit<1>(sfull + 8 * h);
                            if (w.tile(i) == w.half[h].to - 1) mma_commit<1>(qempty + 8 * h);
                        } else if (before[h] && w.tile(i - 1) == w.half[h].to - 1) {
                            mma_commit<1>(ofull + 8 * h);
                        }
                    }
                    before[h] = now;
                }
                if (issuer && ok) mma_commit<1>(empty + 8 * r.slot);
                issued = true;
                r.next();
            }
        }
        if (!ok && issuer) give_up(gave_up, A.err);
    } else if (warp >= 4) {
        const int h = (warp - 4) >> 2, quad = warp & 3;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16, scores = tmem + lanes + h * N, outputs = tmem + lanes + 2 * N + h * 64 * C;
        unsigned char* stage = sm + L::kOut + (warp - 4) * 4096;
        uint32_t tiles = 0, outs = 0;      // so far
        bool ok = true;
        Place w;
        for (int n = 0; ok && place_of(A, n, 2 * N, w); ++n) {
            const int first = w.q0 + h * N, row0 = first + quad * 32, row = row0 + lane;
            const Span mine = span_of(A.sight, first, min(first + N, w.length));
            float followed = -INFINITY;        // the maximum that P is relative to, in powers of two
            float2 total = make_float2(0.f, 0.f);
            bool any = false;
            for (int t = mine.sinks ? 0 : mine.from; t < mine.to; t = t + 1 == mine.sinks ? mine.from : t + 1) {
                ok = R.wait(sfull + 8 * h, tiles & 1);
                if (!ok) break;
                ++tiles;
                tc_fence_after();
                uint32_t s[N];
#pragma unroll
                for (int c = 0; c < N; c += 32) tmem_ld32(scores + c, s + c);
                tmem_wait();
                if (!all_seen(A.sight, first, t)) {
                    // seen: columns up to `near`, and of these the ones after `far` or before `open`, as bits
                    const int near = row - t * N, far = near - A.sight.window, open = A.sight.sinks - t * N;
#pragma unroll
                    for (int c = 0; c < N; c += 32) {
                        const uint32_t bits = low_bits(near + 1 - c) & (~low_bits(far + 1 - c) | low_bits(open - c));
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[c + e] = bits & 1u << e ? s[c + e] : 0xff800000u;
                    }
                }
                float most[4] = {__uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2]), __uint_as_float(s[3])};
#pragma unroll
                for (int c = 4; c < N; c += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most[e] = c + 4 + e < N ? fmaxf(fmaxf(most[e], __uint_as_float(s[c + e])), __uint_as_float(s[c + 4 + e]))
                                                                        : fmaxf(most[e], __uint_as_float(s[c + e]));
                const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * A.scale2;
                if (__any_sync(~0u, top > followed + kGrowth)) {
                    const float now = fmaxf(top, followed), shrink = power(followed - (now == -INFINITY ? 0.f : now));
                    followed = now;
                    total.x *= shrink;
                    total.y *= shrink;
                    if (any) {
#pragma unroll 1
                        for (int c = 0; c < 64 * C; c += 16) {
                            float o[16];
                            tmem_ld(outputs + c, o);
                            tmem_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= shrink;
                            tmem_st(outputs + c, o);
                        }
                    }
                }
                any = true;
                const float less = followed == -INFINITY ? 0.f : kShift - followed;
                const float2 scale = make_float2(A.scale2, A.scale2), minus = make_float2(less, less);
                // in two parts, the first of which is multiplied while the second is computed
#pragma unroll
                for (int c = 0; c < N; c += 64) {
                    uint32_t p[32];
#pragma unroll
                    for (int e = 0; e < 64; e += 2) {
                        float2 x = fma2(make_float2(__uint_as_float(s[c + e]), __uint_as_float(s[c + e + 1])), scale, minus);
                        x.x = power(x.x);
                        x.y = power(x.y);
                        total = add2(total, x);
                        p[e / 2] = pack2<T>(x.x, x.y);
                    }
                    tmem_st32(scores + c / 2, p);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ready + 16 * h + c / 8);
                }
            }
            if (!ok) break;
            if (any) {
                ok = R.wait(ofull + 8 * h, outs & 1);
                if (!ok) break;
                ++outs;
                tc_fence_after();
            }
            const float sum = total.x + total.y;
            const bool in = row < w.length;
            const float inverse = sum == 0.f ? 0.f : 1.f / sum;
            const int rows = min(32, A.sight.tokens - row0);
            T* to_row = static_cast<T*>(A.o) + (((int64_t)w.b * A.sight.tokens + row0) * A.heads + w.head) * (int64_t)A.dim;
            const int64_t pitch = (int64_t)A.heads * A.dim;
#pragma unroll 1
            for (int c = 0; c < 64 * C; c += 64) {
                uint32_t o[64], packed[32];
                tmem_ld32(outputs + c, o);      // (whatever it holds, where the half has no rows)
                tmem_ld32(outputs + c + 32, o + 32);
                tmem_wait();
#pragma unroll
                for (int e = 0; e < 64; e += 2) {
                    const bool real = any && in;
                    packed[e / 2] = pack2<T>(real ? __uint_as_float(o[e]) * inverse : 0.f, real ? __uint_as_float(o[e + 1]) * inverse : 0.f);
                }
                if (A.dim % 8 == 0) {
                    rows_out(stage, packed, reinterpret_cast<char*>(to_row + c), pitch * 2, rows, A.dim - c, lane);
                } else if (lane < rows) {
                    T* to = to_row + lane * pitch + c;
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (c + e < A.dim) reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(packed[e / 2] >> 16 * (e & 1));
                }
            }
            if (A.saved && lane < rows)
                A.saved[((int64_t)w.b * A.heads + w.head) * A.sight.tokens + row] = in ? (followed - kShift + log2f(sum)) * kLn2 : -INFINITY;
        }
        if (!ok && lane == 0) give_up(gave_up, A.err);
    }
    if (warp == 1 && issued) {      // nothing is in flight when tensor memory goes back
        if (issuer) mma_commit<1>(drain);
        mbar_wait(drain, 0, kWaitNs, nullptr);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*gave_up) {
        if (warp == 0) {
            for (int h = 0; h < 2; ++h)
                if (queries[h]) mbar_wait(qfull + 8 * h, (queries[h] - 1) & 1, kWaitNs, nullptr);
            for (uint32_t a = asked > NS ? asked - NS : 0; a < asked; ++a)
                if (!mbar_wait(full + 8 * (a % NS), a / NS & 1, kWaitNs, nullptr)) break;
        }
        __syncthreads();
    }
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(512) : "memory");
}

// Backward.  Both kernels have one shape: 128 resident rows (queries: Q and dO; keys: K and V) and units of 128 rows of
// the other side that stream by (X and Y: K and V, or Q and dO):
//   S = R1 X^T, dP = R2 Y^T
//   P = exp(scale S - lse), dS = P (dP - d), put back as 16-bit elements where S and dP lay
//   queries: dQ += dS X      keys: dV += P Y, dK += dS X
// With keys resident S is the transposed one, so that P and dS are the left operands of their products as they
// lie in tensor memory; lse and d of the columns come with the unit.  Warps 4..7 work on a unit's first 64 columns,
// 8..11 on the others.  One set of S and dP is enough (two would not fit beside dK and dV): while P is computed
// the tensor cores multiply with the last unit's dS and make this unit's dP, and while dS is computed they multiply
// with P and make the next unit's S:
//   keys:    .. dV(u) S(u+1) | dK(u) dP(u+1) ..      queries: .. S(u+1) | dQ(u) dP(u+1) ..
// A 128 x 128 x 16 product takes 64 cycles with its left operand in tensor memory and about 100 with both in shared
// memory, which the left one is read from once for every 64 columns.  So the resident rows lie in tensor memory
// where there is room (queries, and keys of heads up to 64 elements; beside dK and dV of 128 there is none).
// P and dS are rounded to the operands' type.  float16 holds P times 2^14 and
// dS times the power of two that keeps its largest possible value, 2 max|dO| max|V| (row norms), below 2^15: gradients
// of any size keep their bits.
//
// 4 x 4096 tokens as above: 662 us, 1040 TFLOP/s of five products (seven are made); tensor pipe active for 70%.
//
// Keys that stay visible through a window are seen by all later queries: their tiles' far queries are cut into
// pieces, a CTA each, whose sums are joined in their order.
constexpr int kUnit = N;
constexpr float kBackShift = 14.f;         // of float16's P, in powers of two

template <int C, bool kKeys> struct BackShape {
    static constexpr bool kInTmem = !kKeys || C == 1;      // the resident rows
    static constexpr int kTile = C * kChunk;
    static constexpr int kStagesX = C == 2 ? 3 : 4, kStagesY = C == 2 ? 2 : 3;
    static constexpr int kX = kInTmem ? 0 : 2 * kTile, kY = kX + kStagesX * kTile;
    static constexpr int kLse = kY + kStagesY * kTile, kD = kLse + kStagesX * 512;      // of 128 columns for each stage
    static constexpr int kBars = kD + kStagesY * 512;
    static constexpr int kSmem = kBars + 256;
};

struct TcBack {
    CUtensorMap q, k, v, g;
    Heads rows[4];               // the same as they lie in memory: q, k, v, g
    Heads resident[2];           // of them, those whose rows are resident
    View sight;
    const float *lse, *d;        // [batch, heads, pitch]: kBackShift - log2 of the sum (-infinity behind a sequence), and -d
    const float* most;           // float16: largest row norms of dO and V
    void *gq, *gk, *gv;          // dense; for keys' tiles that are cut:
    float* part;                 // [tile][piece][batch * groups][2][128][64 C]
    unsigned* err;
    unsigned long long wait_ns;
    int64_t pitch;
    int tiles, planes;           // of 128 resident rows; heads (groups) of all sequences
    int cut, pieces, piece;      // keys: tiles that are cut, pieces behind the first, queries of one (0: even parts of all units)
    float scale, scale2;
    int heads, groups, dim, width;       // width: elements of a head in memory (copies: a multiple of 8)
};

// 2^k of float16's dS
__device__ __forceinline__ float float16_factor(const float* most) {
    const float bound = 2.f * sqrtf(most[0]) * sqrtf(most[1]);
    if (!(bound > 0.f) || !(bound < 3e38f)) return 1.f;
    int e;
    frexpf(bound, &e);      // bound < 2^e
    return ldexpf(1.f, 15 - e);
}

template <typename T, int C, bool kKeys> __global__ void __launch_bounds__(kThreads, 1) back_tc(const __grid_constant__ TcBack A) {
    using L = BackShape<C, kKeys>;
    constexpr bool kInTmem = L::kInTmem;
    constexpr int NX = L::kStagesX, NY = L::kStagesY;
    constexpr bool kF16 = !std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ __align__(1024) unsigned char sm[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + L::kBars);
    const uint32_t xfull = smem_u32(bars), xempty = xfull + 8 * NX, yfull = xempty + 8 * NX, yempty = yfull + 8 * NY, rfull = yempty + 8 * NY, sfull = rfull + 8,
                   pready = sfull + 8, dpfull = pready + 8, dsready = dpfull + 8, done = dsready + 8, drain = done + 8;
    volatile int* gave_up = reinterpret_cast<volatile int*>(bars + 2 * NX + 2 * NY + 8);
    uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + 2 * NX + 2 * NY + 9);
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t base = smem_u32(sm);

    if (tid == 0) {
        for (int i = 0; i < NX; ++i) {
            mbar_init(xfull + 8 * i, 1);
            mbar_init(xempty + 8 * i, 1);
        }
        for (int i = 0; i < NY; ++i) {
            mbar_init(yfull + 8 * i, 1);
            mbar_init(yempty + 8 * i, 1);
        }
        mbar_init(rfull, kInTmem ? 8 : 1);
        mbar_init(sfull, 1);
        mbar_init(pready, 8);
        mbar_init(dpfull, 1);
        mbar_init(dsready, 8);
        mbar_init(done, 1);
        mbar_init(drain, 1);
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        tma_prefetch(&A.q);
        tma_prefetch(&A.k);
        tma_prefetch(&A.v);
        tma_prefetch(&A.g);
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tslot)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr uint32_t tmem = 0;
    stream_order();

    // The CTA's tile, long ones first: queries from the end; keys: pieces of cut tiles, then the tiles from the start.
    const int per = A.heads / A.groups, which = blockIdx.x % A.planes, row_heads = kKeys ? A.groups : A.heads;
    int tile = blockIdx.x / A.planes, piece = 0;
    if (kKeys) {
        if (!A.piece && A.cut) {
            piece = tile % (A.pieces + 1);
            tile /= A.pieces + 1;
        } else if (tile < A.cut * A.pieces) {
            piece = 1 + tile % A.pieces;
            tile /= A.pieces;
        } else {
            tile -= A.cut * A.pieces;
        }
    } else {
        tile = A.tiles - 1 - tile;
    }
    const int b = which / row_heads, own = which - b * row_heads, length = __shfl_sync(~0u, A.sight.length(b), 0), r0 = tile * N;
    const bool cut = kKeys && tile < A.cut;
    // The units: queries: keys [0, sinks) and [from, to); keys: queries [from, to), of each head of the group.
    int sinks = 0, from = 0, to = 0;
    if (r0 < length) {
        if constexpr (kKeys) {
            // past the window of all, in whole units
            const int near = (int)min(((int64_t)r0 + N + min(A.sight.window, A.sight.tokens) + kUnit - 1) / kUnit * kUnit, (int64_t)1 << 30);
            const bool far = cut && A.piece, all = (r0 < A.sight.sinks || A.sight.window > A.sight.tokens) && !far;
            int first = r0, last = all ? length : min(length, far ? near : min(r0 + N, length) - 1 + A.sight.window);
            if (piece && A.piece) {
                first = near + (piece - 1) * A.piece;
                last = min(length, first + A.piece);
            }
            from = first / kUnit;
            to = last > first ? (last + kUnit - 1) / kUnit : from;
        } else {
            const Span keys = span_of(A.sight, r0, min(r0 + N, length));
            sinks = keys.sinks;
            from = keys.from;
            to = keys.to;
        }
    }
    const int span = sinks + to - from;
    int units = kKeys ? span * per : span, unit0 = 0;
    if (cut && !A.piece) {
        unit0 = (int)((int64_t)units * piece / (A.pieces + 1));
        units = (int)((int64_t)units * (piece + 1) / (A.pieces + 1)) - unit0;
    }
    // first row of a unit, and its head
    auto row_of = [&](int u) {
        const int i = kKeys ? (unit0 + u) % span : u;
        return (i < sinks ? i : from + i - sinks) * kUnit;
    };
    auto head_of = [&](int u) { return kKeys ? own * per + (unit0 + u) / span : own / per; };
    const int tail = length < A.sight.tokens ? length % kUnit : 0;

    const Roles R{gave_up, A.wait_ns};
    const bool issuer = elect_one();
    uint32_t asked_x = 0, asked_y = 0;
    bool issued = false;
    if (warp == 0) {
        bool ok = true;
        if (units && issuer && !kInTmem) {
            mbar_expect(rfull, 2 * L::kTile);
            for (int o = 0; o < 2; ++o)
                for (int c = 0; c < C; ++c) tma_load4(base + o * L::kTile + c * kChunk, kKeys ? (o ? &A.v : &A.k) : (o ? &A.g : &A.q), 64 * c, r0, own, b, rfull);
        }
        Ring<NX> x;
        Ring<NY> y;
        for (int u = 0; u < units; ++u) {
            const int row = row_of(u), head = head_of(u);
            const int64_t at = ((int64_t)b * A.heads + head) * A.pitch + row;
            ok = R.wait_free(xempty + 8 * x.slot, x.phase ^ 1);
            if (!ok) break;
            if (issuer) {
                const uint32_t bar = xfull + 8 * x.slot;
                mbar_expect(bar, L::kTile + (kKeys ? 512 : 0));
                for (int c = 0; c < C; ++c) tma_load4(base + L::kX + x.slot * L::kTile + c * kChunk, kKeys ? &A.q : &A.k, 64 * c, row, head, b, bar);
                if (kKeys) bulk_load(base + L::kLse + x.slot * 512, A.lse + at, 512, bar);
            }
            ++asked_x;
            x.next();
            ok = R.wait_free(yempty + 8 * y.slot, y.phase ^ 1);
            if (!ok) break;
            if (issuer) {
                const uint32_t bar = yfull + 8 * y.slot;
                mbar_expect(bar, L::kTile + (kKeys ? 512 : 0));
                for (int c = 0; c < C; ++c) tma_load4(base + L::kY + y.slot * L::kTile + c * kChunk, kKeys ? &A.g : &A.v, 64 * c, row, head, b, bar);
                if (kKeys) bulk_load(base + L::kD + y.slot * 512, A.d + at, 512, bar);
            }
            ++asked_y;
            y.next();
        }
        let_next();
        if (!ok && issuer) give_up(gave_up, A.err);
    } else if (warp == 1) {
        constexpr uint32_t kType = kF16 ? 0u : 1u << 7 | 1u << 10;
        const uint32_t scores = 1u << 4 | kType | (uint32_t)(N >> 3) << 17 | (uint32_t)(N >> 4) << 24;
        const uint32_t outputs = 1u << 4 | kType | 1u << 16 | (uint32_t)(64 * C >> 3) << 17 | (uint32_t)(N >> 4) << 24;
        const uint64_t d1 = smem_desc(base, 0), d2 = smem_desc(base + L::kTile, 0);
        const uint32_t acc1 = tmem + 256, acc2 = tmem + 256 + 64 * C;
        // 128 x 128 from the resident rows (`which` of them) and a streaming tile
        auto score = [&](uint32_t to_cols, int which, uint32_t tile_at) {
            const uint64_t db = smem_desc(tile_at, 0), da = which ? d2 : d1;
#pragma unroll
            for (int j = 0; j < 4 * C; ++j) {
                const uint32_t step = (j / 4 * kChunk + j % 4 * 32) >> 4;
                if (kInTmem) mma_rows(to_cols, tmem + 384 + 64 * which + 8 * j, db + step, scores, j > 0);
                else mma<1>(to_cols, da + step, db + step, scores, j > 0);
            }
        };
        // += of 16-bit columns (first half at `a`, second 64 columns behind) and a streaming tile
        auto product = [&](uint32_t acc, uint32_t a, uint32_t tile_at, bool first) {
            const uint64_t db = smem_desc(tile_at, kChunk);
#pragma unroll
            for (int j = 0; j < kUnit / 16; ++j) mma_rows(acc, a + (j / 4) * 64 + (j % 4) * 8, db + j * (2048 >> 4), outputs, !first || j > 0);
        };
        // a streaming tile has come; rows behind the sequence: what they hold meets zeros in the products
        auto arrived = [&](uint32_t bar, uint32_t phase, int offset, int u) {
            if (!R.wait(bar, phase)) return false;
            if (tail && row_of(u) == length - tail) clear_rows(sm + offset, C, kUnit, tail, lane);
            return true;
        };
        Ring<NX> x, xu;      // the stages of units u + 1 and u
        Ring<NY> y, yu;
        bool ok = units == 0 || R.wait(rfull, 0);
        tc_fence_after();
        auto with_ds = [&](int u) {      // dK or dQ += dS X
            if (!R.wait(dsready, u & 1)) return false;
            tc_fence_after();
            if (issuer) {
                product(acc1, tmem + 128, base + L::kX + xu.slot * L::kTile, u == 0);
                mma_commit<1>(xempty + 8 * xu.slot);
                // (not with dV: d, which lies beside the stage of Y, has been read by all only where dS is there)
                if (kKeys) mma_commit<1>(yempty + 8 * yu.slot);
            }
            xu.next();
            if (kKeys) yu.next();
            return true;
        };
        for (int u = -1; ok && units && u < units; ++u) {
            if (u >= 0) {
                ok = R.wait(pready, u & 1);      // P (queries: S has been read)
                if (!ok) break;
                tc_fence_after();
                if (kKeys) {
                    if (issuer) product(acc2, tmem, base + L::kY + yu.slot * L::kTile, u == 0);
                }
            }
            if (u + 1 < units) {
                ok = arrived(xfull + 8 * x.slot, x.phase, L::kX + x.slot * L::kTile, u + 1);
                if (!ok) break;
                if (issuer) {
                    score(tmem, 0, base + L::kX + x.slot * L::kTile);
                    mma_commit<1>(sfull);
                }
                issued = true;
                x.next();
            }
            if (u >= 0 && !(ok = with_ds(u))) break;
            if (u + 1 < units) {
                ok = arrived(yfull + 8 * y.slot, y.phase, L::kY + y.slot * L::kTile, u + 1);
                if (!ok) break;
                if (issuer) {
                    score(tmem + 128, 1, base + L::kY + y.slot * L::kTile);
                    mma_commit<1>(dpfull);
                    if (!kKeys) mma_commit<1>(yempty + 8 * y.slot);
                }
                y.next();
            }
        }
        if (issuer) {
            if (!ok) give_up(gave_up, A.err);
            else if (units) mma_commit<1>(done);
        }
    } else if (warp >= 4) {
        const int h = (warp - 4) >> 2, quad = warp & 3, row0 = r0 + quad * 32, row = row0 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16, ts = tmem + lanes + 64 * h, tdp = ts + 128;
        const float factor = kF16 ? float16_factor(A.most) : 1.f;      // of dS
        const float2 scale = make_float2(A.scale2, A.scale2), times = make_float2(factor * 6.103515625e-05f, factor * 6.103515625e-05f);   // 2^-14
        float2 less, minus;       // of a resident query
        if (!kKeys) {
            const int64_t at = ((int64_t)b * A.heads + own) * A.pitch + row;
            less.x = less.y = A.lse[at];
            minus.x = minus.y = A.d[at];
        }
        bool ok = true;
        if (kInTmem && units) {      // a row per lane, as the left operands of products lie there
            const Heads& from_rows = A.resident[h];
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const T*>(from_rows.p) + (int64_t)b * from_rows.batch + (int64_t)row * from_rows.token + (int64_t)own * from_rows.head);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                uint32_t v[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 w = row < A.sight.tokens && 64 * c + 8 * i < A.width ? p[8 * c + i] : make_uint4(0, 0, 0, 0);
                    v[4 * i] = w.x; v[4 * i + 1] = w.y; v[4 * i + 2] = w.z; v[4 * i + 3] = w.w;
                }
                tmem_st32(tmem + lanes + 384 + 64 * h + 32 * c, v);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(rfull);
        }
        Ring<NX> x;
        Ring<NY> y;
        for (int u = 0; u < units; ++u) {
            const int c0 = row_of(u) + 64 * h;      // this thread's first column
            // (lse came with the unit's tile, which the scores were made of; d below as well)
            ok = R.wait(sfull, u & 1);
            if (!ok) break;
            tc_fence_after();
            uint32_t s[64];
            tmem_ld32(ts, s);
            tmem_ld32(ts + 32, s + 32);
            tmem_wait();
            if (!kKeys) {      // the next unit's S may come
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready);
            }
            uint32_t bits[2] = {~0u, ~0u};
            bool some;        // of the columns are not seen by some row
            if (kKeys) {
                some = r0 + N - 1 > c0 || !(c0 + 63 - r0 < A.sight.window || r0 + N - 1 < A.sight.sinks) || c0 + 64 > length;
                if (some) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        bits[c] = ~low_bits(row - c0 - 32 * c) & low_bits(length - c0 - 32 * c) & (row < A.sight.sinks ? ~0u : low_bits(row - c0 - 32 * c + A.sight.window));
                }
            } else {
                some = c0 + 63 > r0 || !(r0 + N - 1 - c0 < A.sight.window || c0 + 63 < A.sight.sinks);
                if (some) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        bits[c] = low_bits(row + 1 - c0 - 32 * c) & (~low_bits(row - A.sight.window + 1 - c0 - 32 * c) | low_bits(A.sight.sinks - c0 - 32 * c));
                }
            }
            const float4* lse = reinterpret_cast<const float4*>(sm + L::kLse + x.slot * 512 + 256 * h);
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
                float4 l;
                if (kKeys) l = lse[c / 4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    if (kKeys) less = e ? make_float2(l.z, l.w) : make_float2(l.x, l.y);
                    const float2 v = fma2(make_float2(__uint_as_float(s[c + e]), __uint_as_float(s[c + e + 1])), scale, less);
                    s[c + e] = __float_as_uint(power(v.x));
                    s[c + e + 1] = __float_as_uint(power(v.y));
                }
            }
            if (some) {
#pragma unroll
                for (int c = 0; c < 64; ++c) s[c] = bits[c / 32] & 1u << c % 32 ? s[c] : 0u;
            }
            if (kKeys) {
                uint32_t p[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) p[c] = pack2<T>(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1]));
                tmem_st32(ts, p);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready);
            }
            ok = R.wait(dpfull, u & 1);
            if (!ok) break;
            tc_fence_after();
            uint32_t p[64];
            tmem_ld32(tdp, p);
            tmem_ld32(tdp + 32, p + 32);
            tmem_wait();
            const float4* d = reinterpret_cast<const float4*>(sm + L::kD + y.slot * 512 + 256 * h);
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
                float4 m;
                if (kKeys) m = d[c / 4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    if (kKeys) minus = e ? make_float2(m.z, m.w) : make_float2(m.x, m.y);
                    const float2 v = make_float2(__uint_as_float(s[c + e]), __uint_as_float(s[c + e + 1]));
                    const float2 w = mul2(kF16 ? mul2(v, times) : v, add2(make_float2(__uint_as_float(p[c + e]), __uint_as_float(p[c + e + 1])), minus));
                    p[c + e] = __float_as_uint(w.x);
                    p[c + e + 1] = __float_as_uint(w.y);
                }
            }
            if (some) {      // (dP of what is not seen may be anything)
#pragma unroll
                for (int c = 0; c < 64; ++c) p[c] = bits[c / 32] & 1u << c % 32 ? p[c] : 0u;
            }
#pragma unroll
            for (int c = 0; c < 32; ++c) s[c] = pack2<T>(__uint_as_float(p[2 * c]), __uint_as_float(p[2 * c + 1]));
            tmem_st32(tdp, s);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(dsready);
            x.next();
            y.next();
        }
        if (ok && units) ok = R.wait(done, 0);
        if (ok) {
            tc_fence_after();
            // keys: dK by the first four warps, dV by the others; queries: 64 columns each
            const bool values = kKeys && h, real = units && row < length;
            const float times_out = values ? (kF16 ? 6.103515625e-05f : 1.f) : A.scale / factor;
            const int rows = min(32, A.sight.tokens - row0);
            unsigned char* stage = sm + L::kX + (warp - 4) * 4096;      // all products are done: the rings are free
            T* to_rows = static_cast<T*>(kKeys ? (h ? A.gv : A.gk) : A.gq) + (((int64_t)b * A.sight.tokens + row0) * row_heads + own) * (int64_t)A.dim;
            const int64_t pitch = (int64_t)row_heads * A.dim;
            float* part = nullptr;
            if (cut) part = A.part + ((((int64_t)tile * (A.pieces + 1) + piece) * A.planes + which) * 2 + h) * N * 64 * C + quad * 32 * 64 * C;
#pragma unroll 1
            for (int c = kKeys ? 0 : 64 * h; c < (kKeys ? 64 * C : 64 * min(C, h + 1)); c += 64) {
                uint32_t o[64];
                tmem_ld32(tmem + lanes + 256 + (values ? 64 * C : 0) + c, o);
                tmem_ld32(tmem + lanes + 256 + (values ? 64 * C : 0) + c + 32, o + 32);
                tmem_wait();
#pragma unroll
                for (int e = 0; e < 64; ++e) o[e] = real ? __float_as_uint(__uint_as_float(o[e]) * times_out) : 0u;
                uint32_t v[32];
                if (cut) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = o[32 * j + e];
                        rows_out(stage, v, reinterpret_cast<char*>(part + c + 32 * j), 64 * C * 4, 32, 64, lane);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = pack2<T>(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
                    if (A.dim % 8 == 0) {
                        rows_out(stage, v, reinterpret_cast<char*>(to_rows + c), pitch * 2, rows, A.dim - c, lane);
                    } else if (lane < rows) {
                        uint16_t* to_row = reinterpret_cast<uint16_t*>(to_rows + lane * pitch + c);
#pragma unroll
                        for (int e = 0; e < 64; ++e)
                            if (c + e < A.dim) to_row[e] = (uint16_t)(v[e / 2] >> 16 * (e & 1));
                    }
                }
            }
        } else if (lane == 0) {
            give_up(gave_up, A.err);
        }
    }
    if (warp == 1 && issued) {      // nothing is in flight when tensor memory goes back
        if (issuer) mma_commit<1>(drain);
        mbar_wait(drain, 0, kWaitNs, nullptr);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*gave_up) {
        if (warp == 0 && units) {
            if (!kInTmem) mbar_wait(rfull, 0, kWaitNs, nullptr);
            for (uint32_t a = asked_x > NX ? asked_x - NX : 0; a < asked_x; ++a)
                if (!mbar_wait(xfull + 8 * (a % NX), a / NX & 1, kWaitNs, nullptr)) break;
            for (uint32_t a = asked_y > NY ? asked_y - NY : 0; a < asked_y; ++a)
                if (!mbar_wait(yfull + 8 * (a % NY), a / NY & 1, kWaitNs, nullptr)) break;
        }
        __syncthreads();
    }
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(512) : "memory");
}

// What the backward needs of each row: -g . o and -lse in powers of two, with float16's shift of P (-infinity behind a
// sequence: no probability), 16 lanes a row, and for float16 the largest squared norms of g's and v's rows.  Bound by HBM.
// o is the rounded one: the sum of p (g . v) over the keys would have to be made by two more products.  Its rounding is one of dS where
// values are about as large as their differences (bfloat16 dQ 0.0025 of its norm, with the unrounded o 0.0025; two keys a row 0.0038 and
// 0.0035), and grows with a part that all values share, which dP - d loses: ten times as large, 0.027 and 0.007.
struct RowArgs {
    Heads g, v;
    const void* o;
    const float* saved;
    float *lse, *d, *most;       // most: [2], or NULL
    const int32_t* lengths;
    int64_t batch, tokens, pitch;
    float shift;
    int heads, groups, dim, packs;
};
__device__ __forceinline__ float sum16(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
template <typename T> __device__ __forceinline__ void load8(const T* p, int c, int dim, int packs, float2 (&v)[4]) {
    if (packs) {
        const uint4 q = c < dim ? *reinterpret_cast<const uint4*>(p + c) : make_uint4(0, 0, 0, 0);
        v[0] = unpack2<T>(q.x); v[1] = unpack2<T>(q.y); v[2] = unpack2<T>(q.z); v[3] = unpack2<T>(q.w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = make_float2(c + 2 * i < dim ? to_f(p[c + 2 * i]) : 0.f, c + 2 * i + 1 < dim ? to_f(p[c + 2 * i + 1]) : 0.f);
    }
}
__device__ __forceinline__ float dot8(const float2 (&a)[4], const float2 (&b)[4]) {
    float2 s = mul2(a[0], b[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = fma2(a[i], b[i], s);
    return s.x + s.y;
}
template <typename T> __global__ void __launch_bounds__(256) rows_tc_kernel(const __grid_constant__ RowArgs A) {
    stream_order();
    const int c = 8 * (threadIdx.x & 15);
    const int64_t step = (int64_t)gridDim.x * 16, rows = A.batch * A.pitch * A.heads, values = A.most ? A.batch * A.tokens * A.groups : 0;
    float most[2] = {0.f, 0.f};
    // Rows in the order of memory, [batch, pitch, heads]: a row's place moves on by a step without divisions.
    // (A warp's two rows stay together: a pitch is a multiple of 128.)
    int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), bt = i / A.heads, b = bt / A.pitch, t = bt - b * A.pitch;
    int h = (int)(i - bt * A.heads);
    const int64_t far = step / A.heads;
    const int more = (int)(step - far * A.heads);
    for (; i < rows; i += step) {
        const bool in = t < (A.lengths ? min(max((int64_t)A.lengths[b], (int64_t)0), A.tokens) : A.tokens);
        const int64_t at = (b * A.heads + h) * A.pitch + t;
        float s = 0.f, n = 0.f, l = 0.f;
        if (in) {
            float2 g[4], o[4];
            load8(static_cast<const T*>(A.g.p) + b * A.g.batch + t * A.g.token + h * A.g.head, c, A.dim, A.packs, g);
            load8(static_cast<const T*>(A.o) + ((b * A.tokens + t) * A.heads + h) * A.dim, c, A.dim, A.packs, o);
            if (c == 0) l = A.saved[(b * A.heads + h) * A.tokens + t];
            s = dot8(g, o);
            n = dot8(g, g);
        }
        s = sum16(s);
        if (A.most) most[0] = fmaxf(most[0], sum16(n));
        if (c == 0) {
            A.d[at] = in ? -s : 0.f;
            A.lse[at] = in ? fmaf(l, -1.44269504088896341f, A.shift) : -INFINITY;
        }
        h += more;
        t += far;
        if (h >= A.heads) {
            h -= A.heads;
            ++t;
        }
        while (t >= A.pitch) {
            t -= A.pitch;
            ++b;
        }
    }
    if (!A.most) return;
    for (int64_t i0 = (int64_t)blockIdx.x * 16; i0 < values; i0 += step) {
        const int64_t i = i0 + (threadIdx.x >> 4), b = i / (A.tokens * A.groups), j = i - b * A.tokens * A.groups, t = j / A.groups;
        const bool in = i < values && t < (A.lengths ? min(max((int64_t)A.lengths[b], (int64_t)0), A.tokens) : A.tokens);
        float n = 0.f;
        if (in) {
            float2 v[4];
            load8(static_cast<const T*>(A.v.p) + b * A.v.batch + t * A.v.token + (j - t * A.groups) * A.v.head, c, A.dim, A.packs, v);
            n = dot8(v, v);
        }
        most[1] = fmaxf(most[1], sum16(n));
    }
    // the largest of non-negative floats as integers: in any order the same (NaN counts as none, an infinity switches the factor off)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float v = fmaxf(most[k], __shfl_xor_sync(~0u, most[k], 16));
        if ((threadIdx.x & 31) == 0) atomicMax(reinterpret_cast<int*>(A.most + k), __float_as_int(v));
    }
}

// Sums of the pieces of cut tiles, in their order: keys and values [tiles * 128 rows] of every group.
template <typename T> __global__ void __launch_bounds__(256) join_tc_kernel(const __grid_constant__ TcBack A, int width) {
    stream_order();
    const int across = (A.dim + 3) / 4, rows = min(A.cut * N, A.sight.tokens);
    const int64_t count = (int64_t)A.planes * 2 * rows * across, step = (int64_t)gridDim.x * 256, plane = (int64_t)A.planes * 2 * N * width;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < count; e += step) {
        const int64_t i = e / across, j = i / rows;
        const int c = (int)(e - i * across) * 4, row = (int)(i - j * rows), side = (int)(j & 1), which = (int)(j >> 1), tile = row / N;
        const float* p = A.part + (int64_t)tile * (A.pieces + 1) * plane + (((int64_t)which * 2 + side) * N + row % N) * width + c;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k <= A.pieces; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(p + k * plane);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const int64_t b = which / A.groups;
        T* to = static_cast<T*>(side ? A.gv : A.gk) + ((b * A.sight.tokens + row) * A.groups + which % A.groups) * A.dim + c;
        if (A.dim % 4 == 0) {
            *reinterpret_cast<uint2*>(to) = make_uint2(pack2<T>(s.x, s.y), pack2<T>(s.z, s.w));
        } else {
            const float v[4] = {s.x, s.y, s.z, s.w};
            for (int k = 0; k < 4 && c + k < A.dim; ++k) to[k] = from_f<T>(v[k]);
        }
    }
}

// Map of heads [batch, tokens, heads, dim]: boxes of 64 elements x `rows` tokens of one head.
bool make_map(CUtensorMap* m, const Heads& h, int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t dim, int rows) {
    EncodeTiled enc = encode_tiled();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)batch};
    // (the stride of an axis of one is not used: any that the driver takes)
    const cuuint64_t strides[3] = {(cuuint64_t)(tokens > 1 ? h.token * 2 : 16), (cuuint64_t)(heads > 1 ? h.head * 2 : 16), (cuuint64_t)(batch > 1 ? h.batch * 2 : 16)};
    const cuuint32_t boxes[4] = {64, (cuuint32_t)rows, 1, 1}, one[4] = {1, 1, 1, 1};
    return enc(m, dtype == VQC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(h.p), dims, strides, boxes, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Heads that TMA cannot read in place (rows off 16-byte boundaries, or one place of memory for several tokens,
// heads or sequences) are copied: dense, rows of a multiple of 8 elements.
struct CopyJob {
    Heads from;
    uint16_t* to;
    int64_t rows;      // batch * tokens * heads
    int heads;
};
struct CopyJobs {
    CopyJob j[4];
    int64_t tokens;
    int dim, padded;
};
__global__ void __launch_bounds__(256) copy_heads_kernel(const __grid_constant__ CopyJobs J) {
    stream_order();
    const CopyJob& A = J.j[blockIdx.y];
    const int across = J.padded / 8;
    const int64_t count = A.rows * across, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < count; e += step) {
        const int64_t row = e / across, bt = row / A.heads, b = bt / J.tokens;
        const int c = (int)(e - row * across) * 8;
        const uint16_t* p = static_cast<const uint16_t*>(A.from.p) + b * A.from.batch + (bt - b * J.tokens) * A.from.token + (row - bt * A.heads) * A.from.head + c;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (c + 2 * i < J.dim ? (uint32_t)p[2 * i] : 0u) | (c + 2 * i + 1 < J.dim ? (uint32_t)p[2 * i + 1] << 16 : 0u);
        *reinterpret_cast<uint4*>(A.to + row * J.padded + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

int64_t padded(int64_t dim) { return (dim + 7) / 8 * 8; }
// On 16-byte boundaries, all heads of all tokens (the stride of an axis of one is not used).
bool on16(const Heads& h, int64_t batch, int64_t tokens, int64_t heads) {
    return aligned_to(h.p, 16) && (batch == 1 || h.batch % 8 == 0) && (tokens == 1 || h.token % 8 == 0) && (heads == 1 || h.head % 8 == 0);
}
bool in_place(const Heads& h, int64_t batch, int64_t tokens, int64_t heads, int64_t dim) {
    constexpr int64_t kMost = int64_t(1) << 38;      // elements: strides of maps have 40 bits of bytes
    auto stride = [](int64_t size, int64_t s) { return size == 1 || (s > 0 && s < kMost); };
    return dim % 8 == 0 && on16(h, batch, tokens, heads) && stride(batch, h.batch) && stride(tokens, h.token) && stride(heads, h.head);
}
size_t copy_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t dim) { return align256((size_t)(batch * tokens * heads) * padded(dim) * 2); }

// Maps of the operands, after copies of those that need one into `ws`.
// (`placed`, where given: the operands as they are read.)
vqc_status maps_of(const AttentionArgs& a, const Heads* const* from, const int* heads, CUtensorMap* const* map, int count, int box, char*& ws, size_t& bytes,
                   Heads* placed, cudaStream_t s) {
    CopyJobs jobs{};
    jobs.tokens = a.sight.tokens;
    jobs.dim = a.dim;
    jobs.padded = (int)padded(a.dim);
    int copies = 0;
    int64_t rows = 0;
    for (int i = 0; i < count; ++i) {
        Heads h = *from[i];
        int64_t dim = a.dim;
        if (!in_place(h, a.batch, a.sight.tokens, heads[i], a.dim)) {
            const size_t need = copy_bytes(a.batch, a.sight.tokens, heads[i], a.dim);
            if (need > bytes) return set_error(VQC_ERR_WORKSPACE, "attention: workspace too small");
            CopyJob& j = jobs.j[copies++];
            j = {h, reinterpret_cast<uint16_t*>(ws), a.batch * a.sight.tokens * heads[i], heads[i]};
            dim = jobs.padded;
            h = {ws, a.sight.tokens * heads[i] * dim, heads[i] * dim, dim};
            rows = std::max(rows, j.rows);
            ws += need;
            bytes -= need;
        }
        if (placed) placed[i] = h;
        if (!make_map(map[i], h, a.dtype, a.batch, a.sight.tokens, heads[i], dim, box)) return set_error(VQC_ERR_CUDA, "attention: a tensor map was refused");
    }
    if (!copies) return VQC_OK;
    void* args[] = {&jobs};
    const int64_t blocks = std::min<int64_t>(ceil_div(rows * (jobs.padded / 8), 256), 8LL * sm_count());
    const cudaError_t e = launch((const void*)copy_heads_kernel, dim3((unsigned)blocks, copies), 256, args, s);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "copy launch");
}

template <typename A> vqc_status start(const AttentionArgs& a, A& t) {
    t.sight = {a.sight.lengths, (int)a.sight.tokens, (int)a.sight.window, (int)a.sight.sinks};
    t.scale = a.scale;
    t.scale2 = a.scale2;
    t.heads = a.heads; t.groups = a.groups; t.dim = a.dim;
    t.wait_ns = wait_limit();
    const cudaError_t e = error_word(&t.err);
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "error word");
}

template <typename T, int C> cudaError_t launch_forward(const TcAttention& t, unsigned grid, cudaStream_t s) {
    void* args[] = {const_cast<TcAttention*>(&t)};
    return launch((const void*)forward_tc<T, C>, dim3(grid), kThreads, args, s, ForwardShape<C>::kSmem);
}

template <typename T, int C, bool kKeys> cudaError_t launch_back(const TcBack& t, cudaStream_t s) {
    void* args[] = {const_cast<TcBack*>(&t)};
    const int64_t tiles = t.tiles + (kKeys ? (int64_t)t.cut * t.pieces : 0);      // (even parts: tiles * (pieces + 1) as well)
    return launch((const void*)back_tc<T, C, kKeys>, dim3((unsigned)(tiles * t.planes)), kThreads, args, s, BackShape<C, kKeys>::kSmem);
}
template <typename T, int C> cudaError_t run_back(TcBack& t, const AttentionArgs& a, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    if (a.gk) {
        t.planes = (int)(a.batch * a.groups);
        t.resident[0] = t.rows[1];
        t.resident[1] = t.rows[2];
        e = launch_back<T, C, true>(t, s);
        if (e == cudaSuccess && t.cut) {
            int width = 64 * C;
            void* args[] = {&t, &width};
            const int64_t count = (int64_t)t.planes * 2 * t.cut * N * (width / 4);
            e = launch((const void*)join_tc_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(count, 256), 8LL * sm_count())), 256, args, s);
        }
    }
    if (e == cudaSuccess && a.gq) {
        t.planes = (int)(a.batch * a.heads);
        t.resident[0] = t.rows[0];
        t.resident[1] = t.rows[3];
        e = launch_back<T, C, false>(t, s);
    }
    return e;
}

// The space of a backward behind the copies: stats of rows, float16's norms, sums of pieces.
struct BackSpace {
    int64_t pitch;
    int cut, pieces, piece;
    size_t stats, most, part;
};
BackSpace back_space(int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t window, int64_t sinks) {
    BackSpace b{};
    b.pitch = ceil_div(tokens, N) * N;
    b.stats = align256((size_t)(batch * heads * b.pitch) * 4);
    b.most = dtype == VQC_F16 ? 256 : 0;
    // Few tiles of keys leave SMs idle: each is cut into even parts of its units, of which every head has about half as
    // many as there are tiles.  (1 x 2048 tokens, 8 heads over one, bfloat16: 172 us in one part, 98 in 2, 61 in 4, 43 in 8, 41 in 16.)
    const int64_t tiles = ceil_div(tokens, N), all = tiles * batch * groups, sms = sm_count();
    if (2 * all <= sms) {
        b.pieces = (int)std::min<int64_t>(std::min<int64_t>(sms / all, 8), std::max<int64_t>(1, heads / groups * (tiles + 1) / 4)) - 1;
        b.cut = b.pieces ? (int)tiles : 0;
        b.part = align256((size_t)b.cut * (b.pieces + 1) * batch * groups * 2 * N * (dim <= 64 ? 64 : 128) * 4);
        return b;
    }
    // Keys seen from behind the window: pieces as long as a window, 2048 queries at least (a piece writes its sums as floats), and no
    // more of them than two CTAs for each SM: that evens the SMs out, and the sums need no more space than 4 such tiles for each (80 MB).
    // (8 heads over 2 of 128, the keys' half, 32768 tokens, 16 first ones, window 256: pieces of 1024 182 us, 2048 174, 4096 264, one 1645.
    // 4096 first tokens, window 1024: 837 us and 143 MB without the bound, 761 with it; over 8 groups, 16000 and 128: 2965 and 2.2 GB, 1783.)
    if (sinks > 0 && window < tokens) {
        const int64_t cut = std::min(ceil_div(sinks, N), tiles), most = 2 * sms / (cut * batch * groups);
        // (where most keys are such there is nothing to even out)
        if (2 * cut > tiles || !most) return b;
        b.cut = (int)cut;
        b.piece = (int)std::max<int64_t>({2048, ceil_div(window + N, kUnit) * kUnit, ceil_div(ceil_div(tokens - window, most), kUnit) * kUnit});
        b.pieces = (int)ceil_div(tokens - window, b.piece);
        b.part = align256((size_t)b.cut * (b.pieces + 1) * batch * groups * 2 * N * (dim <= 64 ? 64 : 128) * 4);
    }
    return b;
}

}  // namespace

bool attention_tc_takes(int dtype, int64_t dim) { return dtype != VQC_F32 && dim <= 128; }

size_t attention_tc_workspace(int mode, int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t window, int64_t sinks,
                              bool aligned) {
    size_t bytes = 0;
    if (!aligned || dim % 8) bytes = (mode ? 2 : 1) * copy_bytes(batch, tokens, heads, dim) + 2 * copy_bytes(batch, tokens, groups, dim);
    if (!mode) return bytes;
    const BackSpace b = back_space(dtype, batch, tokens, heads, groups, dim, window, sinks);
    return bytes + 2 * b.stats + b.most + b.part;
}

vqc_status attention_tc_forward(const AttentionArgs& a, void* ws, size_t bytes, cudaStream_t s) {
    TcAttention t{};
    vqc_status st = start(a, t);
    if (st != VQC_OK) return st;
    const Heads* from[3] = {&a.q, &a.k, &a.v};
    const int heads[3] = {a.heads, a.groups, a.groups};
    CUtensorMap* map[3] = {&t.q, &t.k, &t.v};
    char* at = static_cast<char*>(ws);
    st = maps_of(a, from, heads, map, 3, N, at, bytes, nullptr, s);
    if (st != VQC_OK) return st;
    t.o = a.o;
    t.saved = a.saved;
    t.tiles = (int)ceil_div(a.sight.tokens, 2 * N);
    t.items = (int)(t.tiles * a.batch * a.heads);
    const unsigned grid = (unsigned)std::min<int64_t>(t.items, sm_count());
    const cudaError_t e = a.dtype == VQC_BF16 ? (a.dim <= 64 ? launch_forward<__nv_bfloat16, 1>(t, grid, s) : launch_forward<__nv_bfloat16, 2>(t, grid, s))
                                 : (a.dim <= 64 ? launch_forward<__half, 1>(t, grid, s) : launch_forward<__half, 2>(t, grid, s));
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "attention launch");
}

vqc_status attention_tc_backward(const AttentionArgs& a, void* ws, size_t bytes, cudaStream_t s) {
    TcBack t{};
    vqc_status st = start(a, t);
    if (st != VQC_OK) return st;
    const Heads* from[4] = {&a.q, &a.k, &a.v, &a.g};
    const int heads[4] = {a.heads, a.groups, a.groups, a.heads};
    CUtensorMap* map[4] = {&t.q, &t.k, &t.v, &t.g};
    char* at = static_cast<char*>(ws);
    st = maps_of(a, from, heads, map, 4, N, at, bytes, t.rows, s);
    t.width = (int)padded(a.dim);
    if (st != VQC_OK) return st;
    const BackSpace b = back_space(a.dtype, a.batch, a.sight.tokens, a.heads, a.groups, a.dim, a.sight.window, a.sight.sinks);
    if (2 * b.stats + b.most + b.part > bytes) return set_error(VQC_ERR_WORKSPACE, "attention: workspace too small");
    RowArgs r{};
    r.g = a.g; r.v = a.v;
    r.o = a.o;
    r.saved = a.lse;
    r.lse = reinterpret_cast<float*>(at);
    r.d = reinterpret_cast<float*>(at + b.stats);
    at += 2 * b.stats;
    r.most = b.most ? reinterpret_cast<float*>(at) : nullptr;
    at += b.most;
    r.lengths = a.sight.lengths;
    r.batch = a.batch; r.tokens = a.sight.tokens; r.pitch = b.pitch;
    r.heads = a.heads; r.groups = a.groups; r.dim = a.dim;
    r.shift = a.dtype == VQC_F16 ? kBackShift : 0.f;
    r.packs = a.dim % 8 == 0 && on16(a.g, a.batch, a.sight.tokens, a.heads) && on16(a.v, a.batch, a.sight.tokens, a.groups);
    cudaError_t e = cudaSuccess;
    if (r.most) e = cudaMemsetAsync(r.most, 0, 8, s);
    if (e == cudaSuccess) {
        void* args[] = {&r};
        const int64_t rows = a.batch * a.heads * b.pitch;
        e = launch(a.dtype == VQC_BF16 ? (const void*)rows_tc_kernel<__nv_bfloat16> : (const void*)rows_tc_kernel<__half>,
                   dim3((unsigned)std::min<int64_t>(ceil_div(rows, 16), 12LL * sm_count())), 256, args, s);
    }
    if (e != cudaSuccess) return cuda_error(e, "attention launch");
    t.lse = r.lse;
    t.d = r.d;
    t.most = r.most;
    t.gq = a.gq; t.gk = a.gk; t.gv = a.gv;
    t.part = reinterpret_cast<float*>(at);
    t.pitch = b.pitch;
    t.tiles = (int)ceil_div(a.sight.tokens, N);
    t.cut = b.cut; t.pieces = b.pieces; t.piece = b.piece;
    e = a.dtype == VQC_BF16 ? (a.dim <= 64 ? run_back<__nv_bfloat16, 1>(t, a, s) : run_back<__nv_bfloat16, 2>(t, a, s))
                            : (a.dim <= 64 ? run_back<__half, 1>(t, a, s) : run_back<__half, 2>(t, a, s));
    return e == cudaSuccess ? VQC_OK : cuda_error(e, "attention launch");
}

}  // namespace layers
}  // namespace vqc
