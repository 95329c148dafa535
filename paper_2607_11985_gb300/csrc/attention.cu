// attention.cu -- causal attention through a window and over the first tokens: entry points,
// kernels on the FP32 units for float32 and for 16-bit heads of more than 128 elements.
//
// Query i of a sequence sees key j where j <= i < length and (i - j < window or j < sinks):
//   z_j = scale q . k_j,   lse = log sum_j exp z_j,   o = sum_j exp(z_j - lse) v_j
// and with the incoming gradient g and d = g . o:
//   p_j = exp(z_j - lse),  ds_j = p_j (g . v_j - d),
//   grad_v_j = sum over queries (of all heads that share the key) of p_j g,
//   grad_k_j = scale sum of ds_j q,  grad_q = scale sum_j ds_j k_j.
//
// One pass over the keys: the running maximum and sum of a row are held in float and the row's output is
// rescaled where the maximum grows.  The backward has the tiles' probabilities again from lse, in two
// kernels: one owns keys and sums over queries, one owns queries and sums over keys.  That is seven
// products where five would do with sums across CTAs, but those would need float atomics, whose order
// changes results, or a matrix of partial sums per tile of keys.
//
// Here tiles of 64 queries x 64 keys (32 x 32 for heads of more than 128 elements) lie in shared memory as
// floats, a thread has 4 x 4 scores and 4 rows of the output.  Bound by the reads of shared memory (70% of what it gives) and the FP32
// units (55% of their cycles); 16-bit types with heads up to 128 elements go to the tensor cores (attention_tc.cu).  2 x 2048 tokens, 8
// heads over 2 of 128, float32: forward 460 us (37 TFLOP/s), backward 1690 us (25); of 256, bfloat16: 1660 us (21) and 6650 us (13).
#include <algorithm>
#include <cmath>

#include "attention.h"
#include "layers_elem.cuh"
#include "layers_tc.h"

namespace vqc {
namespace layers {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// Tiles of R rows per thread: 16 R queries x 16 R keys; heads of up to DM elements.
template <int DM> struct Tile {
    static constexpr int R = DM > 128 ? 2 : 4, N = 16 * R;
    static constexpr int kPitch = DM + 4, kScores = N + 4;      // floats between rows: rows 16 apart fall on other banks
    static constexpr int kSmemForward = (2 * N * kPitch + N * kScores) * 4;      // keys and values in turn: two CTAs per SM
    static constexpr int kSmemQueries = (4 * N * kPitch + N * kScores + 2 * N) * 4;
    static constexpr int kSmemKeys = (4 * N * kPitch + 2 * N * kScores + 2 * N) * 4;
};

__device__ __forceinline__ int64_t length_of(const Sight& S, int64_t b) {
    return S.lengths ? min(max((int64_t)S.lengths[b], (int64_t)0), S.tokens) : S.tokens;
}
__device__ __forceinline__ bool sees(const Sight& S, int64_t i, int64_t j, int64_t length) {
    return j <= i && i < length && (i - j < S.window || j < S.sinks);
}

// Rows first.. of one head into shared memory, zeros beyond `rows` and beyond the head's elements.
template <typename T, int DM, int N>
__device__ __forceinline__ void load_tile(float* to, const Heads& x, int64_t b, int64_t head, int64_t first, int64_t rows, int dim) {
    const T* p = static_cast<const T*>(x.p) + b * x.batch + head * x.head;
    if constexpr (sizeof(T) == 4) {
        // floats on 16-byte boundaries: four at a time, straight to their places; all of a thread's are on the way together
        if (dim % 4 == 0 && ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(x.token * 4)) & 15) == 0) {
#pragma unroll
            for (int e = threadIdx.x; e < N * (DM / 4); e += kThreads) {
                const int r = e / (DM / 4), c = e % (DM / 4) * 4;
                const bool in = first + r < rows && c < dim;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"((uint32_t)__cvta_generic_to_shared(to + r * (DM + 4) + c)),
                             "l"(in ? reinterpret_cast<const float*>(p) + (first + r) * x.token + c : reinterpret_cast<const float*>(p)), "r"(in ? 16 : 0)
                             : "memory");
            }
            return;
        }
    }
    for (int e = threadIdx.x; e < N * DM; e += kThreads) {
        const int r = e / DM, c = e % DM;
        to[r * (DM + 4) + c] = first + r < rows && c < dim ? to_f(p[(first + r) * x.token + c]) : 0.f;
    }
}
// The tiles that have been asked for are there, for all threads.
__device__ __forceinline__ void tiles_there() {
    asm volatile("cp.async.wait_all;\n" ::: "memory");
    __syncthreads();
}
// s[i][j] = rows ty R + i of a times rows tx + 16 j of b
template <int DM, int R> __device__ __forceinline__ void scores(const float* a, const float* b, int ty, int tx, float (&s)[R][R]) {
    constexpr int P = DM + 4;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < DM; c += 4) {
        float4 x[R], y[R];
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty * R + i) * P + c);
#pragma unroll
        for (int j = 0; j < R; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * P + c);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j)
                s[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, s[i][j]))));
    }
}
// o[i][c] += sum over k of p[ty R + i][k] v[k][..]: columns 4 tx + 64 c (DM >= 64), or tx + 16 c
template <int DM> constexpr int kOut = DM / 16;
template <int DM> __device__ __forceinline__ int out_col(int tx, int c) { return DM >= 64 ? 4 * tx + 64 * (c / 4) + c % 4 : tx + 16 * c; }
template <int DM, int R> __device__ __forceinline__ void add_product(const float* p, const float* v, int ty, int tx, float (&o)[R][kOut<DM>]) {
    constexpr int P = DM + 4, N = 16 * R, PS = N + 4;
#pragma unroll 2
    for (int k = 0; k < N; k += 4) {
        float4 w[R];
#pragma unroll
        for (int i = 0; i < R; ++i) w[i] = *reinterpret_cast<const float4*>(p + (ty * R + i) * PS + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float row[kOut<DM>];
            if constexpr (DM >= 64) {
#pragma unroll
                for (int c = 0; c < kOut<DM>; c += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(v + (k + e) * P + out_col<DM>(tx, c));
                    row[c] = q.x; row[c + 1] = q.y; row[c + 2] = q.z; row[c + 3] = q.w;
                }
            } else {
#pragma unroll
                for (int c = 0; c < kOut<DM>; ++c) row[c] = v[(k + e) * P + out_col<DM>(tx, c)];
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float x = e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w;
#pragma unroll
                for (int c = 0; c < kOut<DM>; ++c) o[i][c] = fmaf(x, row[c], o[i][c]);
            }
        }
    }
}
template <typename T, int DM, int R>
__device__ __forceinline__ void store_rows(void* to, const float (&o)[R][kOut<DM>], const float (&factor)[R], int64_t at, int64_t pitch, int64_t rows, int dim,
                                           int ty, int tx) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = ty * R + i;
        if (r >= rows) continue;
#pragma unroll
        for (int c = 0; c < kOut<DM>; ++c)
            if (out_col<DM>(tx, c) < dim) static_cast<T*>(to)[at + r * pitch + out_col<DM>(tx, c)] = from_f<T>(o[i][c] * factor[i]);
    }
}
__device__ __forceinline__ float max16(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ float sum16(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// Tiles of keys that queries first..last - 1 may see: [0, sinks) and [from, to), in tiles of N.
struct Span {
    int64_t sinks, from, to;
};
__device__ __forceinline__ Span keys_of(const Sight& S, int64_t first, int64_t last, int N) {
    Span r;
    r.to = (last + N - 1) / N;
    r.from = max((int64_t)0, first - S.window + 1) / N;
    r.sinks = min((min(S.sinks, S.tokens) + N - 1) / N, r.from);
    return r;
}
// one past the last query that sees one of the keys first..last - 1
__device__ __forceinline__ int64_t queries_end(const Sight& S, int64_t first, int64_t last, int64_t length) {
    return first < S.sinks || S.window > S.tokens ? length : min(length, last - 1 + S.window);
}

// The tile of a CTA: (tile, head, sequence), the longest tiles first.
struct At {
    int64_t tile, head, b;
};
__device__ __forceinline__ At tile_of(int64_t tiles, int64_t heads, bool last_first) {
    At r;
    const int64_t plane = (int64_t)gridDim.x / tiles, i = blockIdx.x / plane, j = blockIdx.x - i * plane;
    r.tile = last_first ? tiles - 1 - i : i;
    r.b = j / heads;
    r.head = j - r.b * heads;
    return r;
}

template <typename T, int DM> __global__ void __launch_bounds__(kThreads, 2) forward_kernel(const __grid_constant__ AttentionArgs A, int64_t tiles) {
    stream_order();
    using L = Tile<DM>;
    constexpr int R = L::R, N = L::N;
    extern __shared__ __align__(16) float sm[];
    float *q = sm, *kv = q + N * L::kPitch, *p = kv + N * L::kPitch;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const At W = tile_of(tiles, A.heads, true);
    const int64_t length = length_of(A.sight, W.b), q0 = W.tile * N, q1 = min(q0 + N, length), group = W.head / (A.heads / A.groups);
    float o[R][kOut<DM>], top[R], total[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        top[i] = -INFINITY;
        total[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kOut<DM>; ++c) o[i][c] = 0.f;
    }
    if (q0 < length) {
        load_tile<T, DM, N>(q, A.q, W.b, W.head, q0, length, A.dim);
        const Span span = keys_of(A.sight, q0, q1, N);
        for (int64_t t = span.sinks ? 0 : span.from; t < span.to; t = t + 1 == span.sinks ? span.from : t + 1) {
            __syncthreads();
            load_tile<T, DM, N>(kv, A.k, W.b, group, t * N, length, A.dim);
            tiles_there();
            float s[R][R];
            scores<DM, R>(q, kv, ty, tx, s);
            __syncthreads();
            load_tile<T, DM, N>(kv, A.v, W.b, group, t * N, length, A.dim);      // while the scores are worked on
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float most = top[i];
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    s[i][j] = sees(A.sight, q0 + ty * R + i, t * N + tx + 16 * j, length) ? s[i][j] * A.scale2 : -INFINITY;
                    most = fmaxf(most, s[i][j]);
                }
                most = max16(most);
                const float base = most == -INFINITY ? 0.f : most;      // a row that has seen nothing yet
                const float shrink = exp2f(top[i] - base);
                top[i] = most;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const float e = exp2f(s[i][j] - base);
                    sum += e;
                    p[(ty * R + i) * L::kScores + tx + 16 * j] = e;
                }
                total[i] = total[i] * shrink + sum16(sum);
#pragma unroll
                for (int c = 0; c < kOut<DM>; ++c) o[i][c] *= shrink;
            }
            tiles_there();
            add_product<DM, R>(p, kv, ty, tx, o);
        }
    }
    const int64_t rows = min((int64_t)N, A.sight.tokens - q0);
    if (A.saved && tx == 0) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (ty * R + i < rows)
                A.saved[(W.b * A.heads + W.head) * A.sight.tokens + q0 + ty * R + i] = total[i] > 0.f || total[i] != total[i] ? (top[i] + log2f(total[i])) * kLn2 : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) total[i] = total[i] == 0.f ? 0.f : 1.f / total[i];
    store_rows<T, DM, R>(A.o, o, total, ((W.b * A.sight.tokens + q0) * A.heads + W.head) * A.dim, (int64_t)A.heads * A.dim, rows, A.dim, ty, tx);
}

// d = g . o of every row, a warp each; NaN and infinities stay what they are
template <typename T> __global__ void __launch_bounds__(kThreads) rows_kernel(const __grid_constant__ AttentionArgs A, int64_t rows) {
    stream_order();
    const int lane = threadIdx.x % 32;
    for (int64_t i = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; i < rows; i += (int64_t)gridDim.x * (kThreads / 32)) {
        const int64_t b = i / (A.sight.tokens * A.heads), t = i / A.heads - b * A.sight.tokens, h = i % A.heads;
        if (t >= length_of(A.sight, b)) continue;
        const T* g = static_cast<const T*>(A.g.p) + b * A.g.batch + t * A.g.token + h * A.g.head;
        const T* o = static_cast<const T*>(A.o) + i * A.dim;
        float s = 0.f;
        for (int c = lane; c < A.dim; c += 32) s = fmaf(to_f(g[c]), to_f(o[c]), s);
#pragma unroll
        for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(~0u, s, k);
        if (lane == 0) A.d[(b * A.heads + h) * A.sight.tokens + t] = s;
    }
}

// lse (in powers of two) and d of N rows; rows that are not there see nothing
__device__ __forceinline__ void load_stats(float* lse, float* d, const AttentionArgs& A, const At& W, int64_t head, int64_t first, int64_t length, int N) {
    for (int r = threadIdx.x; r < N; r += kThreads) {
        const int64_t at = (W.b * A.heads + head) * A.sight.tokens + first + r;
        const bool in = first + r < length;
        lse[r] = in ? A.lse[at] * kLog2e : 0.f;
        d[r] = in ? A.d[at] : 0.f;
    }
}

// Gradient of a tile of queries.
template <typename T, int DM> __global__ void __launch_bounds__(kThreads) queries_kernel(const __grid_constant__ AttentionArgs A, int64_t tiles) {
    stream_order();
    using L = Tile<DM>;
    constexpr int R = L::R, N = L::N;
    extern __shared__ __align__(16) float sm[];
    float *q = sm, *g = q + N * L::kPitch, *k = g + N * L::kPitch, *v = k + N * L::kPitch, *ds = v + N * L::kPitch, *lse = ds + N * L::kScores, *d = lse + N;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const At W = tile_of(tiles, A.heads, true);
    const int64_t length = length_of(A.sight, W.b), q0 = W.tile * N, q1 = min(q0 + N, length), group = W.head / (A.heads / A.groups);
    float o[R][kOut<DM>], factor[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        factor[i] = A.scale;
#pragma unroll
        for (int c = 0; c < kOut<DM>; ++c) o[i][c] = 0.f;
    }
    if (q0 < length) {
        load_tile<T, DM, N>(q, A.q, W.b, W.head, q0, length, A.dim);
        load_tile<T, DM, N>(g, A.g, W.b, W.head, q0, length, A.dim);
        load_stats(lse, d, A, W, W.head, q0, length, N);
        const Span span = keys_of(A.sight, q0, q1, N);
        for (int64_t t = span.sinks ? 0 : span.from; t < span.to; t = t + 1 == span.sinks ? span.from : t + 1) {
            __syncthreads();
            load_tile<T, DM, N>(k, A.k, W.b, group, t * N, length, A.dim);
            load_tile<T, DM, N>(v, A.v, W.b, group, t * N, length, A.dim);
            tiles_there();
            float s[R][R], dp[R][R];
            scores<DM, R>(q, k, ty, tx, s);
            scores<DM, R>(g, v, ty, tx, dp);
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const int r = ty * R + i, c = tx + 16 * j;
                    const float e = exp2f(fmaf(s[i][j], A.scale2, -lse[r]));
                    ds[r * L::kScores + c] = sees(A.sight, q0 + r, t * N + c, length) ? e * (dp[i][j] - d[r]) : 0.f;
                }
            __syncwarp();
            add_product<DM, R>(ds, k, ty, tx, o);
        }
    }
    store_rows<T, DM, R>(A.gq, o, factor, ((W.b * A.sight.tokens + q0) * A.heads + W.head) * A.dim, (int64_t)A.heads * A.dim,
                         min((int64_t)N, A.sight.tokens - q0), A.dim, ty, tx);
}

// Gradients of a tile of keys and values: over the heads that share them and the queries that see them.  Where that leaves
// SMs idle (A.part) a CTA takes one of the heads, and sums of the heads are joined in their order.
template <typename T, int DM> __global__ void __launch_bounds__(kThreads) keys_kernel(const __grid_constant__ AttentionArgs A, int64_t tiles) {
    stream_order();
    using L = Tile<DM>;
    constexpr int R = L::R, N = L::N;
    extern __shared__ __align__(16) float sm[];
    float *k = sm, *v = k + N * L::kPitch, *q = v + N * L::kPitch, *g = q + N * L::kPitch, *p = g + N * L::kPitch, *ds = p + N * L::kScores,
          *lse = ds + N * L::kScores, *d = lse + N;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const At W = tile_of(tiles, A.part ? A.heads : A.groups, false);
    const int64_t length = length_of(A.sight, W.b), k0 = W.tile * N, k1 = min(k0 + N, length), per = A.heads / A.groups;
    const int64_t group = A.part ? W.head / per : W.head, h0 = A.part ? W.head : W.head * per, h1 = A.part ? h0 + 1 : h0 + per;
    float gk[R][kOut<DM>], gv[R][kOut<DM>], factor[R], one[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        factor[i] = A.scale;
        one[i] = 1.f;
#pragma unroll
        for (int c = 0; c < kOut<DM>; ++c) gk[i][c] = gv[i][c] = 0.f;
    }
    if (k0 < length) {
        load_tile<T, DM, N>(k, A.k, W.b, group, k0, length, A.dim);
        load_tile<T, DM, N>(v, A.v, W.b, group, k0, length, A.dim);
        const int64_t end = (queries_end(A.sight, k0, k1, length) + N - 1) / N;
        for (int64_t h = h0; h < h1; ++h)
            for (int64_t t = k0 / N; t < end; ++t) {
                __syncthreads();
                load_tile<T, DM, N>(q, A.q, W.b, h, t * N, length, A.dim);
                load_tile<T, DM, N>(g, A.g, W.b, h, t * N, length, A.dim);
                load_stats(lse, d, A, W, h, t * N, length, N);
                tiles_there();
                float s[R][R], dp[R][R];
                scores<DM, R>(k, q, ty, tx, s);
                scores<DM, R>(v, g, ty, tx, dp);
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        const int r = ty * R + i, c = tx + 16 * j;
                        const bool in = sees(A.sight, t * N + c, k0 + r, length);
                        const float e = in ? exp2f(fmaf(s[i][j], A.scale2, -lse[c])) : 0.f;
                        p[r * L::kScores + c] = e;
                        ds[r * L::kScores + c] = in ? e * (dp[i][j] - d[c]) : 0.f;
                    }
                __syncwarp();
                add_product<DM, R>(p, g, ty, tx, gv);
                add_product<DM, R>(ds, q, ty, tx, gk);
            }
    }
    const int64_t rows = min((int64_t)N, A.sight.tokens - k0);
    if (A.part) {      // [2][batch, tokens, heads, dim]
        const int64_t at = ((W.b * A.sight.tokens + k0) * A.heads + W.head) * A.dim, pitch = (int64_t)A.heads * A.dim;
        store_rows<float, DM, R>(A.part, gk, factor, at, pitch, rows, A.dim, ty, tx);
        store_rows<float, DM, R>(A.part + A.batch * A.sight.tokens * pitch, gv, one, at, pitch, rows, A.dim, ty, tx);
        return;
    }
    const int64_t at = ((W.b * A.sight.tokens + k0) * A.groups + W.head) * A.dim, pitch = (int64_t)A.groups * A.dim;
    store_rows<T, DM, R>(A.gk, gk, factor, at, pitch, rows, A.dim, ty, tx);
    store_rows<T, DM, R>(A.gv, gv, one, at, pitch, rows, A.dim, ty, tx);
}

// The heads' sums of each group: [2][rows, heads, dim] to gk and gv [rows, groups, dim].
template <typename T> __global__ void __launch_bounds__(kThreads) join_heads_kernel(const __grid_constant__ AttentionArgs A, int64_t rows) {
    stream_order();
    const int per = A.heads / A.groups;
    const int64_t width = (int64_t)A.groups * A.dim, count = rows * width, step = (int64_t)gridDim.x * kThreads;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < 2 * count; e += step) {
        const int64_t side = e >= count, i = e - side * count, row = i / width;
        const int c = (int)(i - row * width), group = c / A.dim;
        const float* p = A.part + side * rows * A.heads * A.dim + (row * A.heads + (int64_t)group * per) * A.dim + (c - group * A.dim);
        float s = 0.f;
        for (int h = 0; h < per; ++h) s += p[(int64_t)h * A.dim];
        static_cast<T*>(side ? A.gv : A.gk)[i] = from_f<T>(s);
    }
}

template <typename T, int DM> struct Kernels {
    static cudaError_t forward(const AttentionArgs& a0, cudaStream_t s) {
        AttentionArgs a = a0;
        int64_t tiles = ceil_div(a.sight.tokens, Tile<DM>::N);
        void* args[] = {&a, &tiles};
        return launch((const void*)forward_kernel<T, DM>, dim3((unsigned)(tiles * a.batch * a.heads)), kThreads, args, s, Tile<DM>::kSmemForward);
    }
    static cudaError_t queries(const AttentionArgs& a0, cudaStream_t s) {
        AttentionArgs a = a0;
        int64_t tiles = ceil_div(a.sight.tokens, Tile<DM>::N);
        void* args[] = {&a, &tiles};
        return launch((const void*)queries_kernel<T, DM>, dim3((unsigned)(tiles * a.batch * a.heads)), kThreads, args, s, Tile<DM>::kSmemQueries);
    }
    static cudaError_t keys(const AttentionArgs& a0, cudaStream_t s) {
        AttentionArgs a = a0;
        int64_t tiles = ceil_div(a.sight.tokens, Tile<DM>::N);
        void* args[] = {&a, &tiles};
        const cudaError_t e = launch((const void*)keys_kernel<T, DM>, dim3((unsigned)(tiles * a.batch * (a.part ? a.heads : a.groups))), kThreads, args, s, Tile<DM>::kSmemKeys);
        if (e != cudaSuccess || !a.part) return e;
        int64_t rows = a.batch * a.sight.tokens;
        void* join_args[] = {&a, &rows};
        return launch((const void*)join_heads_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(2 * rows * a.groups * a.dim, kThreads), 16LL * sm_count())), kThreads, join_args, s);
    }
    static cudaError_t run(const AttentionArgs& a, int which, cudaStream_t s) { return which == 0 ? forward(a, s) : which == 1 ? queries(a, s) : keys(a, s); }
};
template <typename T> cudaError_t run_typed(const AttentionArgs& a, int which, cudaStream_t s) {
    if constexpr (sizeof(T) == 4) {      // (16-bit heads of up to 128 elements are the tensor cores')
        if (a.dim <= 32) return Kernels<T, 32>::run(a, which, s);
        if (a.dim <= 64) return Kernels<T, 64>::run(a, which, s);
        if (a.dim <= 128) return Kernels<T, 128>::run(a, which, s);
    }
    return Kernels<T, 256>::run(a, which, s);
}
cudaError_t run_plain(const AttentionArgs& a, int which, cudaStream_t s) {
    return a.dtype == VQC_F32 ? run_typed<float>(a, which, s) : a.dtype == VQC_BF16 ? run_typed<__nv_bfloat16>(a, which, s) : run_typed<__half>(a, which, s);
}
cudaError_t rows_run_plain(const AttentionArgs& a0, cudaStream_t s) {
    AttentionArgs a = a0;
    int64_t rows = a.batch * a.sight.tokens * a.heads;
    void* args[] = {&a, &rows};
    const void* fn = a.dtype == VQC_F32 ? (const void*)rows_kernel<float> : a.dtype == VQC_BF16 ? (const void*)rows_kernel<__nv_bfloat16> : (const void*)rows_kernel<__half>;
    return launch(fn, dim3((unsigned)std::min<int64_t>(ceil_div(rows, kThreads / 32), 16LL * sm_count())), kThreads, args, s);
}


vqc_status checked(const char* call, int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t window,
                   int64_t sinks, double scale) {
    if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || !sequence_sizes_ok(batch, tokens, heads, groups) || heads % groups != 0 ||
        dim < 1 || dim > kMostDim)
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": bad type, size, or heads that are no multiple of their groups");
    const float s2 = (float)scale * kLog2e;
    if (window < 0 || sinks < 0 || !(scale > 0) || !std::isnormal(s2))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": a negative window or number of sinks, or a scale that is not positive");
    return VQC_OK;
}
// (tiles of 64 or 32, rows of a warp)
bool grid_ok(int64_t batch, int64_t tokens, int64_t heads, int64_t dim) { return ceil_div(tokens, dim > 128 ? 32 : 64) * batch * heads <= 0x7fffffff; }

AttentionArgs arguments(int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t window, int64_t sinks, double scale,
                        const int32_t* lengths) {
    AttentionArgs a{};
    a.batch = batch; a.heads = (int)heads; a.groups = (int)groups; a.dim = (int)dim; a.dtype = dtype;
    a.sight = {lengths, tokens, window ? std::min(window, kMostTokens + 1) : kMostTokens + 1, std::min(sinks, kMostTokens + 1)};
    a.scale = (float)scale;
    a.scale2 = (float)scale * kLog2e;
    return a;
}
// Space of the heads' sums where the keys' tiles leave SMs idle.
size_t part_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim) {
    if (heads == groups || ceil_div(tokens, dim > 128 ? 32 : 64) * batch * groups >= 2LL * sm_count()) return 0;
    return align256((size_t)(2 * batch * tokens) * heads * dim * 4);
}
size_t saved_bytes(int64_t batch, int64_t tokens, int64_t heads) { return align256((size_t)(batch * tokens) * heads * 4); }

}  // namespace
}  // namespace layers
}  // namespace vqc

using namespace vqc;
using namespace vqc::layers;

extern "C" {

size_t vqc_attention_workspace_bytes(int32_t mode, vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim,
                                     int64_t window, int64_t sinks, int32_t aligned) {
    if ((mode != 0 && mode != 1) || checked("", dtype, batch, tokens, heads, groups, dim, window, sinks, 1.0) != VQC_OK || !grid_ok(batch, tokens, heads, dim))
        return (size_t)-1;
    const Sight s = arguments(dtype, batch, tokens, heads, groups, dim, window, sinks, 1.0, nullptr).sight;
    if (attention_tc_takes(dtype, dim))
        return batch * tokens ? attention_tc_workspace(mode, dtype, batch, tokens, heads, groups, dim, s.window, s.sinks, aligned != 0) : 0;
    return mode ? saved_bytes(batch, tokens, heads) + part_bytes(batch, tokens, heads, groups, dim) : 0;
}

vqc_status vqc_attention_forward(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, const vqc_heads* q,
                                 const vqc_heads* k, const vqc_heads* v, int64_t window, int64_t sinks, double scale, const int32_t* lengths, void* o,
                                 float* saved, void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const char* call = "vqc_attention_forward";
        const vqc_status st = checked(call, dtype, batch, tokens, heads, groups, dim, window, sinks, scale);
        if (st != VQC_OK) return st;
        const size_t e = elem_size(dtype);
        if (!heads_ok(q, e) || !heads_ok(k, e) || !heads_ok(v, e) || (batch * tokens > 0 && (!q->data || !k->data || !v->data || !o)))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL or misaligned operand or output, or a negative stride");
        if (!aligned_to(o, 16) || !aligned_to(saved, 4) || !aligned_to(lengths, 4) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned output, lengths or workspace");
        if (!grid_ok(batch, tokens, heads, dim)) return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": sizes out of range");
        if (batch * tokens == 0) return VQC_OK;
        AttentionArgs a = arguments(dtype, batch, tokens, heads, groups, dim, window, sinks, scale, lengths);
        a.q = heads_of(*q); a.k = heads_of(*k); a.v = heads_of(*v);
        a.o = o;
        a.saved = saved;
        if (attention_tc_takes(dtype, dim)) {
            const vqc_status before = layers_pending();
            return before != VQC_OK ? before : attention_tc_forward(a, workspace, workspace ? workspace_bytes : 0, static_cast<cudaStream_t>(stream));
        }
        const cudaError_t err = run_plain(a, 0, static_cast<cudaStream_t>(stream));
        return err == cudaSuccess ? VQC_OK : cuda_error(err, "attention launch");
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_attention_backward(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, const vqc_heads* grad_o,
                                  const vqc_heads* q, const vqc_heads* k, const vqc_heads* v, const void* o, const float* saved, int64_t window,
                                  int64_t sinks, double scale, const int32_t* lengths, void* grad_q, void* grad_k, void* grad_v, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    try {
        const char* call = "vqc_attention_backward";
        const vqc_status st = checked(call, dtype, batch, tokens, heads, groups, dim, window, sinks, scale);
        if (st != VQC_OK) return st;
        const size_t e = elem_size(dtype);
        if (!heads_ok(grad_o, e) || !heads_ok(q, e) || !heads_ok(k, e) || !heads_ok(v, e) || !grad_k != !grad_v ||
            (batch * tokens > 0 && (!grad_o->data || !q->data || !k->data || !v->data || !o || !saved)))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL or misaligned operand, a negative stride, or one of grad_k and grad_v is NULL");
        if (!aligned_to(o, 16) || !aligned_to(saved, 4) || !aligned_to(lengths, 4) || !aligned_to(grad_q, 16) || !aligned_to(grad_k, 16) ||
            !aligned_to(grad_v, 16) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned output, lengths or workspace");
        if (!grid_ok(batch, tokens, heads, dim)) return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": sizes out of range");
        if (batch * tokens == 0 || (!grad_q && !grad_k)) return VQC_OK;
        const bool tc = attention_tc_takes(dtype, dim);
        if (!workspace || (!tc && workspace_bytes < saved_bytes(batch, tokens, heads) + part_bytes(batch, tokens, heads, groups, dim)))
            return set_error(VQC_ERR_WORKSPACE, std::string(call) + ": workspace too small");
        AttentionArgs a = arguments(dtype, batch, tokens, heads, groups, dim, window, sinks, scale, lengths);
        a.q = heads_of(*q); a.k = heads_of(*k); a.v = heads_of(*v); a.g = heads_of(*grad_o);
        a.o = const_cast<void*>(o);
        a.lse = saved;
        a.d = static_cast<float*>(workspace);
        if (part_bytes(batch, tokens, heads, groups, dim)) a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + saved_bytes(batch, tokens, heads));
        a.gq = grad_q; a.gk = grad_k; a.gv = grad_v;
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        if (tc) {
            const vqc_status before = layers_pending();
            return before != VQC_OK ? before : attention_tc_backward(a, workspace, workspace_bytes, s);
        }
        cudaError_t err = rows_run_plain(a, s);
        if (err == cudaSuccess && grad_k) err = run_plain(a, 2, s);
        if (err == cudaSuccess && grad_q) err = run_plain(a, 1, s);
        return err == cudaSuccess ? VQC_OK : cuda_error(err, "attention launch");
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
