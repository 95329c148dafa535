// attention_cached.cu -- attention of the last tokens of sequences over a cache of keys and values: the
// form for serving, a few queries for many keys.
//
// Token t of a sequence stands at position p = length - tokens + t and sees key j where j <= p and
// (p - j < window or j < sinks); see attention.cu for the formulas.
//
// Bound by HBM: every key and value that is in sight is read once, for all query heads of its group and
// all tokens together.  The keys in sight, [0, sinks) and [from, length) one after the other, are cut
// into chunks, a CTA each; a chunk's maximum, sum and output are joined over the chunks by a second
// launch, in their order.  CTAs beyond a sequence's keys end at once, so that sequences of any mixture of
// lengths keep all SMs busy without the host knowing the lengths.  A token of 24 sequences of up to 8192 keys, 32 heads over 8 of
// 128, bfloat16: 106 us (5.2 TB/s); all of 8192: 140 us (5.7 TB/s).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention.h"
#include "layers_elem.cuh"

namespace vqc {
namespace layers {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr float kLog2e = 1.44269504088896341f;

struct CachedArgs {
    Heads q, k, v;
    const int32_t* lengths;
    int64_t batch, tokens, capacity, window, sinks;
    void* o;
    float *part, *stats;         // [rows][chunks][dim] and [rows][chunks][2], rows (b, head, t), or NULL: one chunk
    float scale2;
    int heads, groups, dim, dtype, chunk, chunks, blocks;      // chunk: keys; blocks of rows of a group
};

// The keys in sight of a sequence's tokens: count, the first ones, and where the rest begins.
struct Keys {
    int64_t length, count, first, from;
};
__device__ __forceinline__ Keys keys_of(const CachedArgs& A, int64_t b) {
    Keys r;
    r.length = min(max((int64_t)A.lengths[b], (int64_t)0), A.capacity);
    r.from = max((int64_t)0, r.length - A.tokens - A.window + 1);
    r.first = min(A.sinks, r.from);
    r.count = r.first + r.length - r.from;
    return r;
}
__device__ __forceinline__ int64_t key_at(const Keys& K, int64_t i) { return i < K.first ? i : K.from + (i - K.first); }

// 16 bytes to shared memory, or zeros; the end of a group of copies; at most M groups still on the way
__device__ __forceinline__ void copy16(void* to, const void* from, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;\n" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int M> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(M) : "memory"); }
template <typename T> __device__ __forceinline__ void as_floats(const uint4& q, float* v) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __uint_as_float(w[i]);
        } else {
            const float2 a = unpack2<T>(w[i]);
            v[2 * i] = a.x;
            v[2 * i + 1] = a.y;
        }
    }
}
constexpr int kDepth = 4;      // groups of keys of a warp, on the way or being worked on

// Any type and head size: 8 lanes hold a key (V elements at a time), 4 keys per warp, RB queries; each of
// the 16 places of a CTA has a maximum, a sum and an output of its own until the chunk ends.
template <typename T, int DM, int V, int RB> __global__ void __launch_bounds__(kThreads) cached_kernel(const __grid_constant__ CachedArgs A) {
    stream_order();
    constexpr int NE = DM / 8, NL = NE / V;      // elements of a lane, loads
    extern __shared__ __align__(16) float joined[];     // the ring, and after it the places' sums
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = warp * 4 + lane / 8, part = lane & 7;
    int64_t w = blockIdx.x;      // all groups of a chunk together: they read neighbouring memory
    const int group = (int)(w % A.groups);
    w /= A.groups;
    const int block = (int)(w % A.blocks);
    w /= A.blocks;
    const int64_t chunk = w % A.chunks, b = w / A.chunks;
    const Keys K = keys_of(A, b);
    const int64_t i0 = chunk * A.chunk, i1 = min(i0 + A.chunk, K.count);
    if (i0 >= i1 && chunk > 0) return;
    const int per = A.heads / A.groups, rows = (int)min((int64_t)RB, per * A.tokens - (int64_t)block * RB);
    auto col = [&](int l, int e) { return (l * 8 + part) * V + e; };
    float q[RB][NE], o[RB][NE], top[RB], total[RB];
    int64_t at[RB];      // position
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t row = (int64_t)block * RB + r, h = group * per + row / A.tokens, t = row % A.tokens;
        const T* p = static_cast<const T*>(A.q.p) + b * A.q.batch + t * A.q.token + h * A.q.head;
        at[r] = r < rows ? K.length - A.tokens + t : -1;
        top[r] = -INFINITY;
        total[r] = 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const int c = col(i / V, i % V);
            q[r][i] = r < rows && c < A.dim ? to_f(p[c]) * A.scale2 : 0.f;
            o[r][i] = 0.f;
        }
    }
    const T *kp = static_cast<const T*>(A.k.p) + b * A.k.batch + group * A.k.head, *vp = static_cast<const T*>(A.v.p) + b * A.v.batch + group * A.v.head;
    // Keys and values on the way: a lane copies the 16 bytes that it will read itself, so that nobody waits for another's
    // (elements that are not there arrive as zeros).  Single elements (V = 1) are loaded when they are needed.
    unsigned char* ring = reinterpret_cast<unsigned char*>(joined) + warp * kDepth * 2 * NL * 512 + lane * 16;
    auto ask = [&](int64_t i, int stage) {
        if constexpr (V > 1) {
            const bool there = i + slot < i1;
            const int64_t j = there ? key_at(K, i + slot) : 0;
#pragma unroll
            for (int l = 0; l < NL; ++l) {
                const bool in = there && col(l, 0) < A.dim;
                copy16(ring + (stage * 2 * NL + l) * 512, in ? kp + j * A.k.token + col(l, 0) : kp, in);
                copy16(ring + (stage * 2 * NL + NL + l) * 512, in ? vp + j * A.v.token + col(l, 0) : vp, in);
            }
            copies_end();
        }
    };
    if (i1 > i0) {
#pragma unroll
        for (int d = 0; d < kDepth - 1; ++d) ask(i0 + 16 * d, d);
    }
    int stage = 0;
    for (int64_t i = i0; i < i1; i += 16) {
        const bool in = i + slot < i1;
        const int64_t j = in ? key_at(K, i + slot) : 0;
        float k[NE], v[NE];
        if constexpr (V > 1) {
            copies_wait<kDepth - 2>();
            const int last = stage ? stage - 1 : kDepth - 1;
#pragma unroll
            for (int l = 0; l < NL; ++l) {
                as_floats<T>(*reinterpret_cast<const uint4*>(ring + (stage * 2 * NL + l) * 512), k + l * V);
                as_floats<T>(*reinterpret_cast<const uint4*>(ring + (stage * 2 * NL + NL + l) * 512), v + l * V);
            }
            ask(i + 16 * (kDepth - 1), last);
            stage = stage + 1 == kDepth ? 0 : stage + 1;
        } else {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                k[e] = in && col(e, 0) < A.dim ? to_f(kp[j * A.k.token + col(e, 0)]) : 0.f;
                v[e] = in && col(e, 0) < A.dim ? to_f(vp[j * A.v.token + col(e, 0)]) : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < NE; ++e) s = fmaf(q[r][e], k[e], s);
            s += __shfl_xor_sync(~0u, s, 1);
            s += __shfl_xor_sync(~0u, s, 2);
            s += __shfl_xor_sync(~0u, s, 4);
            if (!in || j > at[r] || (at[r] - j >= A.window && j >= A.sinks)) continue;      // (the same in a key's 8 lanes)
            if (s > top[r]) {
                const float shrink = exp2f(top[r] - s);
                top[r] = s;
                total[r] *= shrink;
#pragma unroll
                for (int e = 0; e < NE; ++e) o[r][e] *= shrink;
            }
            const float p = exp2f(s - (top[r] == -INFINITY ? 0.f : top[r]));
            total[r] += p;
#pragma unroll
            for (int e = 0; e < NE; ++e) o[r][e] = fmaf(p, v[e], o[r][e]);
        }
        __syncwarp();
    }
    constexpr int P = DM + 2;
    let_next();      // the join may be placed
    if (V > 1) copies_wait<0>();
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RB; ++r) {
#pragma unroll
        for (int i = 0; i < NE; ++i) joined[(r * 16 + slot) * P + col(i / V, i % V)] = o[r][i];
        if (part == 0) {
            joined[(r * 16 + slot) * P + DM] = top[r];
            joined[(r * 16 + slot) * P + DM + 1] = total[r];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * DM; e += kThreads) {
        const int r = e / DM, c = e % DM;
        float most = -INFINITY, sum = 0.f, out = 0.f;
        for (int s = 0; s < 16; ++s) most = fmaxf(most, joined[(r * 16 + s) * P + DM]);
        for (int s = 0; s < 16; ++s) {
            const float* x = joined + (r * 16 + s) * P;
            const float f = x[DM] == -INFINITY && x[DM + 1] == 0.f ? 0.f : exp2f(x[DM] - (most == -INFINITY ? 0.f : most));
            sum += f * x[DM + 1];
            out += f * x[c];
        }
        if (c >= A.dim) continue;
        const int64_t row = (int64_t)block * RB + r, h = group * per + row / A.tokens, t = row % A.tokens;
        if (A.part) {
            const int64_t to = ((b * A.heads + h) * A.tokens + t) * A.chunks + chunk;
            A.part[to * A.dim + c] = out;
            if (c == 0) {
                A.stats[2 * to] = most;
                A.stats[2 * to + 1] = sum;
            }
        } else {
            static_cast<T*>(A.o)[((b * A.tokens + t) * A.heads + h) * A.dim + c] = from_f<T>(sum == 0.f ? 0.f : out / sum);
        }
    }
}

// 16-bit types with heads of up to 128 elements, on the tensor cores' mma.sync (a few rows leave tcgen05's tiles of 128
// empty, and what bounds this is the loads): a warp takes 16 keys at a time for 16 rows (queries of a group, all tokens).
// Both operands go from memory to registers as they lie there.  The scores contract over a head's elements, in
// any order that both operands share: a lane's 16 bytes of a key, elements 32 i + 8 t + [0, 8), are its
// parts of two steps.  The output's columns are free as well: column n of block j is element 64 (j / 8) + 8 n + j % 8, so that
// a lane's 16 bytes of a value are its column in eight blocks; two keys' halves are paired by a byte permutation.
// A lane copies the 16 bytes that it will read itself to shared memory, three stages deep: nobody waits for another's
// copies, and what is on the way takes no registers (in registers 5.2 TB/s).
constexpr int kRows = 16;
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit elements (two neighbours of row g in lane 4 g + t), its rows for its columns
__device__ __forceinline__ uint32_t turned8(uint32_t w) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ float power(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// A stage: the pieces of 16 keys and values of a warp, each where the lane that copied it reads it.
template <int DM, int W> struct MmaShape {
    static constexpr int NK = DM / 32, NV = DM / 64, kPieces = 2 * NK + 4 * NV, kStage = kPieces * 512, kDeep = DM == 64 ? 4 : 3;
    static constexpr int kRing = W * kDeep * kStage, kSums = W * kRows * (DM + 4) * 4;
    static constexpr int kSmem = (kRing > kSums ? kRing : kSums) + W * kRows * 8;
};

// kFew: 8 rows at most.  The products are the transposed ones, S^T = K Q^T and O^T = V^T P^T, with 16 keys (16 elements of a
// value) in the place of the 16 rows: half as many, and half the registers of the output; P^T is turned by movmatrix.  A
// lane then has rows 2 t and 2 t + 1 of keys g and g + 8, and a row's maximum is looked for over the lanes only where
// some key is above the followed one by 2^8.
template <typename T, int DM, int W, bool kFew> __global__ void __launch_bounds__(32 * W, W == 8 ? 1 : DM == 64 ? 4 : 2) cached_mma_kernel(const __grid_constant__ CachedArgs A) {
    using L = MmaShape<DM, W>;
    constexpr int NK = L::NK, NV = L::NV, kDeep = L::kDeep;      // pieces of 16 bytes of a lane: of a key, of a value
    constexpr float kShift = sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value ? 6.f : 0.f;
    constexpr int P = DM + 4;
    extern __shared__ __align__(16) unsigned char shared[];
    float(*joined)[kRows][P] = reinterpret_cast<float(*)[kRows][P]>(shared);      // in the place of the ring, after it
    float(*stats)[kRows][2] = reinterpret_cast<float(*)[kRows][2]>(shared + L::kSmem - W * kRows * 8);
    stream_order();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    int64_t w = blockIdx.x;      // all groups of a chunk together: they read neighbouring memory
    const int group = (int)(w % A.groups);
    w /= A.groups;
    const int block = (int)(w % A.blocks);
    w /= A.blocks;
    const int64_t chunk = w % A.chunks, b = w / A.chunks;
    const Keys K = keys_of(A, b);
    const int64_t i0 = chunk * A.chunk;
    if (i0 >= K.count && chunk > 0) return;
    const int count = (int)max((int64_t)0, min((int64_t)A.chunk, K.count - i0));
    const int per = A.heads / A.groups, tokens = (int)A.tokens, rows = min(kRows, per * tokens - block * kRows);
    const T *kp = static_cast<const T*>(A.k.p) + b * A.k.batch + group * A.k.head, *vp = static_cast<const T*>(A.v.p) + b * A.v.batch + group * A.v.head;
    unsigned char* ring = shared + warp * kDeep * L::kStage + lane * 16;
    // keys and values of index i0 + i behind the first ones
    const T *kq = kp + (K.from - K.first + i0 + g) * A.k.token + 8 * t, *vq = vp + (K.from - K.first + i0 + 2 * t) * A.v.token + 8 * g;
    const uint32_t ring32 = (uint32_t)__cvta_generic_to_shared(ring);
    auto ask = [&](int i, int stage) {
        unsigned char* to = ring + stage * L::kStage;
        if (i + 16 <= count && i0 + i >= K.first && A.dim == DM) {      // nearly always
            const uint32_t to32 = ring32 + stage * L::kStage;
            const T *pk = kq + i * A.k.token, *pv = vq + i * A.v.token;
#pragma unroll
            for (int n = 0; n < 2; ++n, pk += 8 * A.k.token)
#pragma unroll
                for (int c = 0; c < NK; ++c) copy16(to32 + (n * NK + c) * 512, pk + 32 * c);
#pragma unroll
            for (int n = 0; n < 4; ++n, pv += n == 2 ? 7 * A.v.token : A.v.token)
#pragma unroll
                for (int c = 0; c < NV; ++c) copy16(to32 + (2 * NK + n * NV + c) * 512, pv + 64 * c);
            copies_end();
            return;
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int at_i = i + g + 8 * n;
            const T* p = kp + key_at(K, i0 + at_i) * A.k.token + 8 * t;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const bool in = at_i < count && 32 * c + 8 * t < A.dim;
                copy16(to + (n * NK + c) * 512, in ? p + 32 * c : kp, in);
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int at_i = i + 2 * t + (n & 1) + 8 * (n >> 1);
            const T* p = vp + key_at(K, i0 + at_i) * A.v.token + 8 * g;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const bool in = at_i < count && 64 * c + 8 * g < A.dim;
                copy16(to + (2 * NK + n * NV + c) * 512, in ? p + 64 * c : vp, in);
            }
        }
        copies_end();
    };
    constexpr int kStep = 16 * W;
    if (count) {
#pragma unroll
        for (int d = 0; d < kDeep - 1; ++d) ask(16 * warp + d * kStep, d);
    }
    // queries of rows g (and g + 8), while the first keys come; positions of the rows of this lane's scores
    uint32_t q[2 * NK][4];
    int at[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        at[r] = (int)(K.length - tokens) + (block * kRows + (kFew ? 2 * t + r : g + 8 * r)) % tokens;
        if (kFew && r) break;
        const int row = block * kRows + g + 8 * r, h = group * per + row / tokens, tok = row % tokens;
        const bool in = g + 8 * r < rows;
        const T* p = static_cast<const T*>(A.q.p) + b * A.q.batch + tok * A.q.token + h * A.q.head;
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int c = 32 * i + 8 * t;
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {      // (queries may have any alignment)
                const uint32_t lo = in && c < A.dim ? reinterpret_cast<const uint16_t*>(p)[c + 2 * e] : 0u, hi = in && c < A.dim ? reinterpret_cast<const uint16_t*>(p)[c + 2 * e + 1] : 0u;
                x[e] = lo | hi << 16;
            }
            q[2 * i][r] = x[0];
            q[2 * i][2 + r] = x[1];
            q[2 * i + 1][r] = x[2];
            q[2 * i + 1][2 + r] = x[3];
        }
    }
    constexpr int NO = kFew ? 4 * NV : 8 * NV;
    float o[NO][4], followed[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NO; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    int stage = 0;
    for (int i = 16 * warp; i < count; i += kStep) {
        copies_wait<kDeep - 2>();
        const unsigned char* from = ring + stage * L::kStage;
        // all of a stage's pieces at once: one by one, each before its products, their latencies took half of the time
        uint4 kw[2][NK], vw[4][NV];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int c = 0; c < NK; ++c) kw[n][c] = *reinterpret_cast<const uint4*>(from + (n * NK + c) * 512);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int c = 0; c < NV; ++c) vw[n][c] = *reinterpret_cast<const uint4*>(from + (2 * NK + n * NV + c) * 512);
        ask(i + (kDeep - 1) * kStep, stage ? stage - 1 : kDeep - 1);
        stage = stage + 1 == kDeep ? 0 : stage + 1;
        if constexpr (kFew) {
            float s[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};      // two sums side by side
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const uint32_t a0[4] = {kw[0][c].x, kw[1][c].x, kw[0][c].y, kw[1][c].y}, a1[4] = {kw[0][c].z, kw[1][c].z, kw[0][c].w, kw[1][c].w};
                mma_16816(s, a0, q[2 * c][0], q[2 * c][2], T());
                mma_16816(s1, a1, q[2 * c + 1][0], q[2 * c + 1][2], T());
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += s1[e];
            // element e: key i + g + 8 (e / 2), row 2 t + e % 2
            if (tokens > 1 || i + 16 > count) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at_i = i + g + 8 * (e >> 1);
                    bool seen = at_i < count;
                    if (tokens > 1) {      // (one token sees every key that is counted)
                        const int64_t j = key_at(K, i0 + at_i), p = at[e & 1];
                        seen = seen && j <= p && (p - j < A.window || j < A.sinks);
                    }
                    if (!seen) s[e] = -INFINITY;
                }
            }
            float top[2] = {fmaxf(s[0], s[2]) * A.scale2, fmaxf(s[1], s[3]) * A.scale2};
            if (__any_sync(~0u, top[0] > followed[0] + 8.f || top[1] > followed[1] + 8.f)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], x));
                    const float now = fmaxf(followed[r], top[r]), shrink = power(followed[r] - (now == -INFINITY ? 0.f : now));
                    followed[r] = now;
                    total[r] *= shrink;
#pragma unroll
                    for (int j = 0; j < NO; ++j) {
                        o[j][r] *= shrink;
                        o[j][2 + r] *= shrink;
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = followed[e & 1];
                s[e] = power(fmaf(s[e], A.scale2, f == -INFINITY ? 0.f : kShift - f));
                total[e & 1] += s[e];
            }
            const uint32_t p0 = turned8(pack2<T>(s[0], s[1])), p1 = turned8(pack2<T>(s[2], s[3]));
            // block 4 c + j: elements 64 c + 8 g + 2 j (and the one behind it, as rows g + 8 of the left operand)
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const uint32_t v[4][4] = {{vw[0][c].x, vw[0][c].y, vw[0][c].z, vw[0][c].w}, {vw[1][c].x, vw[1][c].y, vw[1][c].z, vw[1][c].w},
                                          {vw[2][c].x, vw[2][c].y, vw[2][c].z, vw[2][c].w}, {vw[3][c].x, vw[3][c].y, vw[3][c].z, vw[3][c].w}};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a[4] = {__byte_perm(v[0][j], v[1][j], 0x5410), __byte_perm(v[0][j], v[1][j], 0x7632), __byte_perm(v[2][j], v[3][j], 0x5410),
                                           __byte_perm(v[2][j], v[3][j], 0x7632)};
                    mma_16816(o[4 * c + j], a, p0, p1, T());
                }
            }
        } else {
            float s[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
            for (int c = 0; c < NK; ++c)
#pragma unroll
                for (int n = 0; n < 2; ++n) {      // (the two sums go on side by side)
                    mma_16816(s[n], q[2 * c], kw[n][c].x, kw[n][c].y, T());
                    mma_16816(s[n], q[2 * c + 1], kw[n][c].z, kw[n][c].w, T());
                }
            // element e of s[n]: row g + 8 (e / 2), key i + 8 n + 2 t + e % 2
            if (tokens > 1 || i + 16 > count)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at_i = i + 8 * n + 2 * t + (e & 1);
                    bool seen = at_i < count;
                    if (tokens > 1) {      // (one token sees every key that is counted)
                        const int64_t j = key_at(K, i0 + at_i), p = at[e >> 1];
                        seen = seen && j <= p && (p - j < A.window || j < A.sinks);
                    }
                    if (!seen) s[n][e] = -INFINITY;
                }
            float top[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1])) * A.scale2;
                top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 1));
                top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 2));
            }
            // the followed maximum moves when it has grown by more than 2^8
            if (__any_sync(~0u, top[0] > followed[0] + 8.f || top[1] > followed[1] + 8.f)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float now = fmaxf(followed[r], top[r]), shrink = power(followed[r] - (now == -INFINITY ? 0.f : now));
                    followed[r] = now;
                    total[r] *= shrink;
#pragma unroll
                    for (int j = 0; j < 8 * NV; ++j) {
                        o[j][2 * r] *= shrink;
                        o[j][2 * r + 1] *= shrink;
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float f = followed[e >> 1];
                    s[n][e] = power(fmaf(s[n][e], A.scale2, f == -INFINITY ? 0.f : kShift - f));
                    total[e >> 1] += s[n][e];
                }
            const uint32_t p[4] = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]),
                                   pack2<T>(s[1][2], s[1][3])};
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                uint32_t v[4][4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    v[n][0] = vw[n][c].x; v[n][1] = vw[n][c].y; v[n][2] = vw[n][c].z; v[n][3] = vw[n][c].w;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t order = j & 1 ? 0x7632 : 0x5410;
                    mma_16816(o[8 * c + j], p, __byte_perm(v[0][j / 2], v[1][j / 2], order), __byte_perm(v[2][j / 2], v[3][j / 2], order), T());
                }
            }
        }
    }
    let_next();      // the join may be placed
    copies_wait<0>();
    __syncthreads();
    if constexpr (kFew) {      // row 2 t + r, element 64 c + 8 g + 2 j + k of o[4 c + j][2 k + r]
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) total[r] += __shfl_xor_sync(~0u, total[r], x);
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int j = 0; j < 4; j += 2)
                    *reinterpret_cast<float4*>(&joined[warp][2 * t + r][64 * c + 8 * g + 2 * j]) = make_float4(o[4 * c + j][r], o[4 * c + j][2 + r], o[4 * c + j + 1][r], o[4 * c + j + 1][2 + r]);
            if (g == 0) {
                stats[warp][2 * t + r][0] = followed[r];
                stats[warp][2 * t + r][1] = total[r];
            }
        }
    } else {
        // a warp's sums to shared memory: row g + 8 r, element 64 c + 8 n + j of o[8 c + j][2 r + n % 2], n = 2 t, 2 t + 1
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            total[r] += __shfl_xor_sync(~0u, total[r], 1);
            total[r] += __shfl_xor_sync(~0u, total[r], 2);
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int j = 0; j < 8; j += 4)
                        *reinterpret_cast<float4*>(&joined[warp][g + 8 * r][64 * c + 16 * t + 8 * n + j]) =
                            make_float4(o[8 * c + j][2 * r + n], o[8 * c + j + 1][2 * r + n], o[8 * c + j + 2][2 * r + n], o[8 * c + j + 3][2 * r + n]);
            if (t == 0) {
                stats[warp][g + 8 * r][0] = followed[r];
                stats[warp][g + 8 * r][1] = total[r];
            }
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * (DM / 4); e += 32 * W) {
        const int r = e / (DM / 4), c = e % (DM / 4) * 4;
        if (c >= A.dim) continue;      // (dim is a multiple of 8)
        float most = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) most = fmaxf(most, stats[k][r][0]);
        float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const float f = stats[k][r][0] == -INFINITY ? (stats[k][r][1] == 0.f ? 0.f : 1.f) : power(stats[k][r][0] - most);
            const float4 x = *reinterpret_cast<const float4*>(&joined[k][r][c]);
            sum += f * stats[k][r][1];
            out.x += f * x.x; out.y += f * x.y; out.z += f * x.z; out.w += f * x.w;
        }
        const int row = block * kRows + r;
        const int64_t h = group * per + row / tokens, tok = row % tokens;
        if (A.part) {
            const int64_t to = ((b * A.heads + h) * tokens + tok) * A.chunks + chunk;
            *reinterpret_cast<float4*>(A.part + to * A.dim + c) = out;
            if (c == 0) {
                A.stats[2 * to] = most;
                A.stats[2 * to + 1] = sum;
            }
        } else {
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            *reinterpret_cast<uint2*>(static_cast<T*>(A.o) + ((b * tokens + tok) * A.heads + h) * A.dim + c) = make_uint2(pack2<T>(out.x * f, out.y * f), pack2<T>(out.z * f, out.w * f));
        }
    }
}

// A row's chunks joined, in an order of their own: by a warp (kWarpsOfRow 1), or where there are many by 8 warps, which take every
// 8th chunk.
template <typename T, int kWarpsOfRow> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ CachedArgs A, int64_t rows) {
    stream_order();
    constexpr int kCols = kMostDim / 32;
    __shared__ float sums[8][kMostDim], weights[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = kWarpsOfRow == 1 ? blockIdx.x * 8ll + warp : blockIdx.x, t = row % A.tokens, h = row / A.tokens % A.heads, b = row / A.tokens / A.heads;
    if (row >= rows) return;
    const Keys K = keys_of(A, b);
    const int chunks = (int)max((int64_t)1, (K.count + A.chunk - 1) / A.chunk), first = kWarpsOfRow == 1 ? 0 : warp;
    const float* stats = A.stats + 2 * row * A.chunks;
    float most = -INFINITY;
    for (int c = lane; c < chunks; c += 32) most = fmaxf(most, stats[2 * c]);
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    float out[kCols], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kCols; ++i) out[i] = 0.f;
#pragma unroll 4
    for (int c = first; c < chunks; c += kWarpsOfRow) {
        const float m = stats[2 * c], l = stats[2 * c + 1];
        const float f = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(m - most);
        sum += f * l;
        const float* p = A.part + (row * A.chunks + c) * A.dim;
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (lane + 32 * i < A.dim) out[i] += f * p[lane + 32 * i];
    }
    T* o = static_cast<T*>(A.o) + ((b * A.tokens + t) * A.heads + h) * A.dim;
    if constexpr (kWarpsOfRow == 1) {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (lane + 32 * i < A.dim) o[lane + 32 * i] = from_f<T>(out[i] * f);
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i) sums[warp][lane + 32 * i] = out[i];
        if (lane == 0) weights[warp] = sum;
        __syncthreads();
        for (int c = threadIdx.x; c < A.dim; c += 256) {
            float v = 0.f, total = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v += sums[i][c];
                total += weights[i];
            }
            o[c] = from_f<T>(total == 0.f ? 0.f : v / total);
        }
    }
}
template <typename T> const void* join_fn(bool wide) { return wide ? (const void*)join_kernel<T, 8> : (const void*)join_kernel<T, 1>; }

// A kernel and its shared memory.
struct Chosen {
    const void* fn;
    size_t shared;
};
template <typename T, int DM, int RB> Chosen cached_fn(bool packs) {
    constexpr int V = 16 / sizeof(T), W = DM / 8 >= V ? V : 1;
    constexpr size_t sums = 16 * RB * (DM + 2) * 4, ring = (size_t)kWarps * kDepth * 2 * (DM / 8 / W) * 512;
    if constexpr (W > 1 && (sizeof(T) == 4 || DM > 128))      // (packs of 16-bit heads of up to 128 elements are cached_mma_kernel's)
        if (packs) return {(const void*)cached_kernel<T, DM, W, RB>, std::max(sums, ring)};
    return {(const void*)cached_kernel<T, DM, 1, RB>, sums};
}
template <typename T> Chosen cached_fn(int dim, bool packs) {
    return dim <= 32 ? cached_fn<T, 32, 4>(packs) : dim <= 64 ? cached_fn<T, 64, 4>(packs) : dim <= 128 ? cached_fn<T, 128, 4>(packs) : cached_fn<T, 256, 2>(packs);
}
template <typename T, int W, bool kFew> Chosen cached_mma_fn(int dim) {
    if (dim <= 64) return {(const void*)cached_mma_kernel<T, 64, W, kFew>, MmaShape<64, W>::kSmem};
    return {(const void*)cached_mma_kernel<T, 128, W, kFew>, MmaShape<128, W>::kSmem};
}
template <typename T> Chosen cached_mma_fn(int dim, bool one, bool few) {
    if (few) return one ? cached_mma_fn<T, 8, true>(dim) : cached_mma_fn<T, kWarps, true>(dim);
    return one ? cached_mma_fn<T, 8, false>(dim) : cached_mma_fn<T, kWarps, false>(dim);
}

// How the keys are cut.  `most`: keys that can be in sight at once.  The chunks of one, two, .. waves of CTAs that the SMs
// hold together are compared by their longest SM: its keys, and for each CTA the time of about 192 keys to begin and to
// end.  Sequences of a batch have other lengths, which the host does not know: the same for two thirds of the
// keys, dealt as SMs get free, counts twice.  (There is a token at least.)
// What the numbers are worth, in us of a pass alone with flushed caches, sequences of up to 8192 keys of other lengths: without the 192 keys
// 16 of 16 heads over 4 of 64 elements take 66 (38), with 384 of them 24 of 32 heads over 8 of 128 take 144 (124).  Without the half
// chunk at the end those take 145, and 16 float32 ones of 8 heads of 128 188 (155).  Two thirds: a half is the same, the whole takes 169 for
// the floats.  Other sizes change by less than 8%.
struct Cut {
    int chunk, chunks, blocks;
    size_t part, stats;      // bytes
};
constexpr int kOne = 1024;
Cut cut_of(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity, int64_t window, int64_t sinks, bool mma) {
    Cut c{};
    const int64_t most = window ? std::min(capacity, std::min(window, kMostTokens) + tokens - 1 + std::min(sinks, kMostTokens)) : capacity;
    c.blocks = (int)ceil_div(heads / groups * tokens, mma ? kRows : dim > 128 ? 2 : 4);
    // (A few keys are one CTA's of 8 warps: the second launch takes longer than 128 keys of a warp.)
    if (mma && most <= kOne) {
        c.chunk = kOne;
        c.chunks = 1;
        return c;
    }
    const int64_t units = batch * groups * c.blocks, wave = (int64_t)sm_count() * (mma && dim <= 64 ? 4 : 2), least = 64;
    double best = 1e300;
    for (int waves = 1; waves <= 16; ++waves) {
        const int64_t chunks = std::max<int64_t>(1, std::min(ceil_div(most, least), waves * wave / units));
        const int64_t chunk = std::max(least, ceil_div(ceil_div(most, chunks), 16) * 16);
        const int64_t ctas = ceil_div(most, chunk) * units;
        double cost = (double)ceil_div(ctas, wave) * (chunk + 192);
        if (batch > 1) cost += 2 * (ctas <= wave ? chunk + 192.0 : 0.67 * ctas / wave * (chunk + 192) + 0.5 * chunk);
        if (cost < best) {
            best = cost;
            c.chunk = (int)chunk;
        }
    }
    c.chunks = (int)std::max<int64_t>(1, ceil_div(most, c.chunk));
    if (c.chunks > 1) {
        const size_t rows = (size_t)batch * heads * tokens * c.chunks;
        c.part = align256(rows * dim * 4);
        c.stats = align256(rows * 8);
    }
    return c;
}
// (Rows (b, head, token) within 31 bits: no more CTAs than that, as a block has a row at least, and cut_of makes no more chunks of blocks
// than stay on the SMs in 16 waves.)
bool sizes_ok(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity) {
    return sequence_sizes_ok(batch, tokens, heads, groups) && heads % groups == 0 && batch * tokens * heads <= 0x7fffffff && dim >= 1 && dim <= kMostDim &&
           capacity >= 0 && capacity <= kMostTokens;
}

}  // namespace
}  // namespace layers
}  // namespace vqc

using namespace vqc;
using namespace vqc::layers;

extern "C" {

size_t vqc_attention_step_workspace_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity, int64_t window,
                                          int64_t sinks) {
    if (!sizes_ok(batch, tokens, heads, groups, dim, capacity) || window < 0 || sinks < 0) return (size_t)-1;
    if (batch * tokens == 0) return 0;
    // (the most of the two kernels, one of which the cache's alignment decides on)
    const Cut c = cut_of(batch, tokens, heads, groups, dim, capacity, window, sinks, false), m = cut_of(batch, tokens, heads, groups, dim, capacity, window, sinks, true);
    return std::max(c.part + c.stats, m.part + m.stats);
}

vqc_status vqc_attention_step(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity,
                              const vqc_heads* q, const vqc_heads* cache_k, const vqc_heads* cache_v, int64_t window, int64_t sinks, double scale,
                              const int32_t* lengths, void* o, void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const std::string call = "vqc_attention_step";
        if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || !sizes_ok(batch, tokens, heads, groups, dim, capacity))
            return set_error(VQC_ERR_INVALID_ARG, call + ": bad type, size, or heads that are no multiple of their groups");
        const float s2 = (float)scale * kLog2e;
        if (window < 0 || sinks < 0 || !(scale > 0) || !std::isnormal(s2))
            return set_error(VQC_ERR_INVALID_ARG, call + ": a negative window or number of sinks, or a scale that is not positive");
        const size_t e = elem_size(dtype);
        if (!heads_ok(q, e) || !heads_ok(cache_k, e) || !heads_ok(cache_v, e) ||
            (batch * tokens > 0 && (!q->data || !lengths || !o || (capacity > 0 && (!cache_k->data || !cache_v->data)))))
            return set_error(VQC_ERR_INVALID_ARG, call + ": NULL or misaligned operand or output, or a negative stride");
        if (!aligned_to(o, 16) || !aligned_to(lengths, 4) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, call + ": misaligned output, lengths or workspace");
        if (batch * tokens == 0) return VQC_OK;
        const bool packs = dim % (16 / (int64_t)e) == 0 && heads_on(heads_of(*cache_k), e, 16) && heads_on(heads_of(*cache_v), e, 16);
        const bool mma = packs && dtype != VQC_F32 && dim <= 128;
        const Cut c = cut_of(batch, tokens, heads, groups, dim, capacity, window, sinks, mma);
        if (c.chunks > 1 && (!workspace || workspace_bytes < c.part + c.stats)) return set_error(VQC_ERR_WORKSPACE, call + ": workspace too small");
        const int64_t grid = batch * groups * c.blocks * c.chunks, rows = batch * heads * tokens;
        CachedArgs a{};
        a.q = heads_of(*q); a.k = heads_of(*cache_k); a.v = heads_of(*cache_v);
        a.lengths = lengths;
        a.batch = batch; a.tokens = tokens; a.capacity = capacity;
        a.window = window ? std::min(window, kMostTokens + 1) : kMostTokens + 1;
        a.sinks = std::min(sinks, kMostTokens + 1);
        a.o = o;
        a.scale2 = s2;
        a.heads = (int)heads; a.groups = (int)groups; a.dim = (int)dim; a.dtype = dtype;
        a.chunk = c.chunk; a.chunks = c.chunks; a.blocks = c.blocks;
        if (c.chunks > 1) {
            a.part = static_cast<float*>(workspace);
            a.stats = reinterpret_cast<float*>(static_cast<char*>(workspace) + c.part);
        }
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        void* args[] = {&a};
        const bool few = heads / groups * tokens <= 8;
        const Chosen fn = mma ? (dtype == VQC_BF16 ? cached_mma_fn<__nv_bfloat16>(a.dim, c.chunks == 1, few) : cached_mma_fn<__half>(a.dim, c.chunks == 1, few)) : dtype == VQC_F32 ? cached_fn<float>(a.dim, packs) : dtype == VQC_BF16 ? cached_fn<__nv_bfloat16>(a.dim, packs) : cached_fn<__half>(a.dim, packs);
        cudaError_t err = launch(fn.fn, dim3((unsigned)grid), mma && c.chunks == 1 ? 256 : kThreads, args, s, fn.shared);
        if (err == cudaSuccess && c.chunks > 1) {
            const bool wide = c.chunks > 4;
            int64_t count = rows;
            void* join_args[] = {&a, &count};
            err = launch(dtype == VQC_F32 ? join_fn<float>(wide) : dtype == VQC_BF16 ? join_fn<__nv_bfloat16>(wide) : join_fn<__half>(wide),
                         dim3((unsigned)(wide ? rows : ceil_div(rows, 8))), 256, join_args, s);
        }
        return err == cudaSuccess ? VQC_OK : cuda_error(err, "cached attention launch");
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
