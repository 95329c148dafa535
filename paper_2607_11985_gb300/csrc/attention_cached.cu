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
// lengths keep all SMs busy without the host knowing the lengths.
#include <algorithm>
#include <cmath>

#include "attention.h"
#include "layers_elem.cuh"

namespace vqc {
namespace layers {

namespace {

constexpr int kThreads = 128;
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

// V elements of a row, as floats
template <typename T, int V> __device__ __forceinline__ void load_some(const T* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = to_f(*p);
    } else {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
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
}

// Any type and head size: 8 lanes hold a key (V elements at a time), 4 keys per warp, RB queries; each of
// the 16 places of a CTA has a maximum, a sum and an output of its own until the chunk ends.
template <typename T, int DM, int V, int RB> __global__ void __launch_bounds__(kThreads) cached_kernel(const __grid_constant__ CachedArgs A) {
    stream_order();
    constexpr int NE = DM / 8, NL = NE / V;      // elements of a lane, loads
    __shared__ float joined[16 * RB * (DM + 2)];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = warp * 4 + lane / 8, part = lane & 7;
    int64_t w = blockIdx.x;
    const int64_t chunk = w % A.chunks;
    w /= A.chunks;
    const int block = (int)(w % A.blocks);
    w /= A.blocks;
    const int group = (int)(w % A.groups);
    const int64_t b = w / A.groups;
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
    for (int64_t i = i0; i < i1; i += 16) {
        const bool in = i + slot < i1;
        const int64_t j = in ? key_at(K, i + slot) : 0;
        float k[NE], v[NE];
#pragma unroll
        for (int l = 0; l < NL; ++l) {
            float x[V], y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = y[e] = 0.f;
            if (in && col(l, 0) < A.dim) {
                load_some<T, V>(kp + j * A.k.token + col(l, 0), x);
                load_some<T, V>(vp + j * A.v.token + col(l, 0), y);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                k[l * V + e] = x[e];
                v[l * V + e] = y[e];
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

// A row's chunks joined: a CTA per row, 8 warps take every 8th chunk.
template <typename T> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ CachedArgs A) {
    stream_order();
    constexpr int kCols = kMostDim / 32;
    __shared__ float sums[8][kMostDim], weights[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x, t = row % A.tokens, h = row / A.tokens % A.heads, b = row / A.tokens / A.heads;
    const Keys K = keys_of(A, b);
    const int chunks = (int)max((int64_t)1, (K.count + A.chunk - 1) / A.chunk);
    const float* stats = A.stats + 2 * row * A.chunks;
    float most = -INFINITY;
    for (int c = lane; c < chunks; c += 32) most = fmaxf(most, stats[2 * c]);
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    float out[kCols], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kCols; ++i) out[i] = 0.f;
    for (int c = warp; c < chunks; c += 8) {
        const float m = stats[2 * c], l = stats[2 * c + 1];
        if (m == -INFINITY && l == 0.f) continue;
        const float f = exp2f(m - (most == -INFINITY ? 0.f : most));
        sum += f * l;
        const float* p = A.part + (row * A.chunks + c) * A.dim;
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (lane + 32 * i < A.dim) out[i] += f * p[lane + 32 * i];
    }
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
        static_cast<T*>(A.o)[((b * A.tokens + t) * A.heads + h) * A.dim + c] = from_f<T>(total == 0.f ? 0.f : v / total);
    }
}

template <typename T, int DM, int RB> const void* cached_fn(bool packs) {
    constexpr int V = 16 / sizeof(T);
    return packs && DM / 8 >= V ? (const void*)cached_kernel<T, DM, (DM / 8 >= V ? V : 1), RB> : (const void*)cached_kernel<T, DM, 1, RB>;
}
template <typename T> const void* cached_fn(int dim, bool packs) {
    return dim <= 32 ? cached_fn<T, 32, 4>(packs) : dim <= 64 ? cached_fn<T, 64, 4>(packs) : dim <= 128 ? cached_fn<T, 128, 4>(packs) : cached_fn<T, 256, 2>(packs);
}

// How the keys are cut.  `most`: keys that can be in sight at once.  Chunks of 64 to 512 keys: short ones where
// there are few rows, so that all SMs take part, long ones where the parts of the output would count.
struct Cut {
    int chunk, chunks, blocks;
    size_t part, stats;      // bytes
};
Cut cut_of(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity, int64_t window, int64_t sinks) {
    Cut c{};
    const int64_t most = window ? std::min(capacity, std::min(window, kMostTokens) + tokens - 1 + std::min(sinks, kMostTokens)) : capacity;
    c.blocks = (int)ceil_div(heads / groups * tokens, dim > 128 ? 2 : 4);
    const int64_t units = batch * groups * c.blocks, even = ceil_div(most * units, 6LL * sm_count());
    c.chunk = (int)std::min<int64_t>(512, std::max<int64_t>(64, ceil_div(even, 64) * 64));
    c.chunks = (int)std::max<int64_t>(1, ceil_div(most, c.chunk));
    if (c.chunks > 1) {
        const size_t rows = (size_t)batch * heads * tokens * c.chunks;
        c.part = align256(rows * dim * 4);
        c.stats = align256(rows * 8);
    }
    return c;
}
bool sizes_ok(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity) {
    return sequence_sizes_ok(batch, tokens, heads, groups) && heads % groups == 0 && dim >= 1 && dim <= kMostDim && capacity >= 0 && capacity <= kMostTokens;
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
    const Cut c = cut_of(batch, tokens, heads, groups, dim, capacity, window, sinks);
    return c.part + c.stats;
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
        const Cut c = cut_of(batch, tokens, heads, groups, dim, capacity, window, sinks);
        if (c.chunks > 1 && (!workspace || workspace_bytes < c.part + c.stats)) return set_error(VQC_ERR_WORKSPACE, call + ": workspace too small");
        const int64_t grid = batch * groups * c.blocks * c.chunks, rows = batch * heads * tokens;
        if (grid > 0x7fffffff || rows > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, call + ": sizes out of range");
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
        const bool packs = dim % (16 / (int64_t)e) == 0 && heads_on(a.k, e, 16) && heads_on(a.v, e, 16);
        void* args[] = {&a};
        const void* fn = dtype == VQC_F32 ? cached_fn<float>(a.dim, packs) : dtype == VQC_BF16 ? cached_fn<__nv_bfloat16>(a.dim, packs) : cached_fn<__half>(a.dim, packs);
        cudaError_t err = launch(fn, dim3((unsigned)grid), kThreads, args, s);
        if (err == cudaSuccess && c.chunks > 1) {
            const void* join = dtype == VQC_F32 ? (const void*)join_kernel<float> : dtype == VQC_BF16 ? (const void*)join_kernel<__nv_bfloat16> : (const void*)join_kernel<__half>;
            err = launch(join, dim3((unsigned)rows), 256, args, s);
        }
        return err == cudaSuccess ? VQC_OK : cuda_error(err, "cached attention launch");
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
