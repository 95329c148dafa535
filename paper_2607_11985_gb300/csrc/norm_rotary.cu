// norm_rotary.cu -- norms of queries and keys for each head, with the position rotation in the same
// pass: forward, backward, and the form for serving that puts keys and values into a cache.
//
//   h = x / sqrt(mean(x^2) + eps) * weight             over a head's elements
//   y_i = h_i cos a - h_{n+i} sin a,  y_{n+i} = h_{n+i} cos a + h_i sin a,   a = position * frequency_i, i < n
// and with g the incoming gradient turned back (a replaced by -a), r = 1 / sqrt(..), m = x r:
//   grad_weight = sum of g m,   grad_x = r (u - m mean(u m)),  u = g weight.
//
// The angle is taken modulo a turn in integers: a frequency is a 64-bit fraction of a turn per
// position, whose product with the position wraps by itself.  What is lost is a double's
// rounding of the frequency (4e-7 of a radian at position 2^31 and frequency 1) and a float's of an argument within half a turn.
//
// Bound by HBM (x once, y once; x and the gradient once, the result once).  A head's elements lie
// in the registers of 4 to 32 lanes, each lane with 4 of the first half and their 4 partners, so that pairs meet
// in a lane; a lane keeps its sines and cosines over the heads of its token.  8192 tokens of 32 + 8 heads of 128, bfloat16:
// forward 33 us (5.1 TB/s), backward 54 (4.6 TB/s): a head's sums wait for its loads, of which the next heads' are on the way, and
// 8192 units of work for the 4864 groups of lanes that stay on the SMs take the time of two rounds.  float32: 58 us (5.8 TB/s), 101 (5.0).
#include <algorithm>
#include <cmath>

#include "layers_elem.cuh"
#include "sequence.h"

namespace vqc {
namespace layers {

namespace {

constexpr int kMostDim = 256, kThreads = 256;

struct Side {
    Heads x, g;           // input, incoming gradient
    Rows y;               // output (forward: y; backward: grad_x)
    const void* weight;   // or NULL
    int heads;
};
struct RotaryArgs {
    Side side[3];              // queries, keys, values (copied; the form for serving)
    const double* frequency;   // [pairs] radians per position
    const int32_t* position;   // [batch or 1][tokens], or NULL: the token's index
    const int32_t* lengths;    // [batch], the form for serving: token t stands at lengths - tokens + t
    int64_t position_stride, batch, tokens, capacity;
    float* part;               // [CTAs][2][dim] sums of the weights' gradients, or NULL
    float eps;
    int dim, pairs, chunk, chunks, copies;       // chunk: heads of a unit of work; chunks of a token
};

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int o = lanes / 2; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// A frequency as a fraction of a turn per position, in 2^-64: a double's mantissa moved to its place (one double product;
// doubles are slow here).
__device__ __forceinline__ uint64_t turn_of(double frequency) {
    const uint64_t u = (uint64_t)__double_as_longlong(frequency * 0.15915494309189533577);      // 1 / 2 pi
    const int biased = (int)(u >> 52 & 0x7ff), up = biased - 1075 + 64;
    const uint64_t m = (u & 0xfffffffffffffull) | (biased ? 1ull << 52 : 0);
    const uint64_t r = up >= 64 || up <= -64 ? 0 : up >= 0 ? m << up : m >> -up;
    return (int64_t)u < 0 ? 0 - r : r;
}
// sin and cos of position * frequency
__device__ __forceinline__ float2 turned(uint64_t turn, int64_t position) {
    const int32_t part = (int32_t)((turn * (uint64_t)position + 0x80000000ull) >> 32);      // 2^-32 of a turn, to nearest
    float2 r;
    sincospif((float)part * 4.65661287307739e-10f, &r.x, &r.y);      // 2^-31
    return r;
}

// 4 elements as they lie in memory, and as two pairs of floats
template <typename T> struct Four {
    uint2 w;
    __device__ __forceinline__ void ask(const T* p) { w = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void get(float2 (&v)[2]) const {
        v[0] = unpack2<T>(w.x);
        v[1] = unpack2<T>(w.y);
    }
};
template <> struct Four<float> {
    float4 w;
    __device__ __forceinline__ void ask(const float* p) { w = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float2 (&v)[2]) const {
        v[0] = make_float2(w.x, w.y);
        v[1] = make_float2(w.z, w.w);
    }
};
template <typename T> __device__ __forceinline__ void store4(T* p, float2 a, float2 b) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(a.x, a.y, b.x, b.y);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(a.x, a.y), pack2<T>(b.x, b.y));
}
__device__ __forceinline__ float2 neg2(float2 a) { return make_float2(-a.x, -a.y); }
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// A unit of work: up to `chunk` heads of one token, by one group of LANES lanes.
struct Unit {
    int64_t b, t, pos;      // pos: the token's position
    int first, last;        // heads, counted over the sides
    bool inside;            // of the cache
};
__device__ __forceinline__ Unit unit_at(const RotaryArgs& A, int64_t u, int total) {
    Unit r;
    // (neighbouring groups of lanes have the same heads of neighbouring tokens: a warp's groups walk the same loops)
    const int64_t tokens = A.batch * A.tokens, token = u % tokens;
    r.first = (int)(u / tokens) * A.chunk;
    r.last = min(total, r.first + A.chunk);
    r.b = token / A.tokens;
    r.t = token - r.b * A.tokens;
    if (A.lengths) {
        r.pos = (int64_t)A.lengths[r.b] - A.tokens + r.t;
        r.inside = r.pos >= 0 && r.pos < A.capacity;
    } else {
        r.pos = A.position ? A.position[r.b * A.position_stride + r.t] : r.t;
    }
    return r;
}
// Where side s of a token is written: dense rows, or a place of the cache (NULL outside of it).
template <typename T> __device__ __forceinline__ T* out_at(const RotaryArgs& A, const Unit& U, int s, int h) {
    const Rows& y = A.side[s].y;
    if (A.lengths && s && !U.inside) return nullptr;
    return static_cast<T*>(y.p) + U.b * y.batch + (A.lengths && s ? U.pos : U.t) * y.token + (int64_t)h * y.head;
}

// Heads in packs of 4 elements: dim a multiple of 8, pairs of 4, all rows on 4-element boundaries.
// Lane j of a group holds the 4 pairs (4j, n + 4j) for 4j < n, or 8 elements that are not turned.
template <typename T, int LANES, bool kBack> __global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryArgs A) {
    stream_order();
    constexpr int kGroups = kThreads / LANES, HB = sizeof(T) == 4 || kBack ? 2 : 4;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, total = A.side[0].heads + A.side[1].heads + A.side[2].heads;
    const uint32_t peers = LANES == 32 ? ~0u : ((1u << (LANES & 31)) - 1) << (threadIdx.x & 31 & ~(LANES - 1));
    const int turning = A.pairs / 4;
    const bool on = lane < A.dim / 8, turns = lane < turning;
    const int ca = turns ? 4 * lane : 2 * A.pairs + 8 * (lane - turning), cb = turns ? A.pairs + 4 * lane : ca + 4;
    const int64_t units = A.batch * A.tokens * A.chunks, step = (int64_t)gridDim.x * kGroups;
    const float per = 1.f / (float)A.dim;
    auto group_sum = [&](float v) {
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(peers, v, o);
        return v;
    };
    uint64_t freq[4] = {0, 0, 0, 0};
    if (turns) {
#pragma unroll
        for (int i = 0; i < 4; ++i) freq[i] = turn_of(A.frequency[4 * lane + i]);
    }
    float2 sum[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[0][i] = sum[1][i] = both(0.f);
    for (int64_t u = (int64_t)blockIdx.x * kGroups + group; u < units; u += step) {
        const Unit U = unit_at(A, u, total);
        float2 cosine[2], sine[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 p = turns ? turned(freq[2 * i], U.pos) : make_float2(0.f, 1.f), q = turns ? turned(freq[2 * i + 1], U.pos) : make_float2(0.f, 1.f);
            sine[i] = make_float2(p.x, q.x);
            cosine[i] = make_float2(p.y, q.y);
        }
        int before = 0;
#pragma unroll
        for (int s = 0; s < (kBack ? 2 : 3); ++s) {
            const Side& S = A.side[s];
            const int lo = max(U.first - before, 0), hi = min(U.last - before, S.heads);
            before += S.heads;
            if (lo >= hi) continue;
            float2 w[4] = {both(1.f), both(1.f), both(1.f), both(1.f)};
            if (S.weight && on) {
                Four<T> p[2];
                float2 v[2];
                p[0].ask(static_cast<const T*>(S.weight) + ca);
                p[1].ask(static_cast<const T*>(S.weight) + cb);
                p[0].get(v);
                w[0] = v[0]; w[1] = v[1];
                p[1].get(v);
                w[2] = v[0]; w[3] = v[1];
            }
            const T *px = static_cast<const T*>(S.x.p) + U.b * S.x.batch + U.t * S.x.token + lo * S.x.head + ca, *pg = nullptr;
            if (kBack) pg = static_cast<const T*>(S.g.p) + U.b * S.g.batch + U.t * S.g.token + lo * S.g.head + ca;
            T* py = out_at<T>(A, U, s, lo);
            const bool writes = py && on && (!kBack || S.y.p);
            py += ca;
            const int other = cb - ca;
            // The next HB heads' elements are asked for before these are worked on: 8 bytes a load alone would leave HBM waiting.
            Four<T> next[HB][kBack ? 4 : 2], these[HB][kBack ? 4 : 2];
            auto ask = [&](int h) {
#pragma unroll
                for (int j = 0; j < HB; ++j) {
                    if (on && h + j < hi) {
                        next[j][0].ask(px);
                        next[j][1].ask(px + other);
                        if constexpr (kBack) {
                            next[j][2].ask(pg);
                            next[j][3].ask(pg + other);
                        }
                    }
                    px += S.x.head;
                    if (kBack) pg += S.g.head;
                }
            };
            ask(lo);
#pragma unroll 1
            for (int h = lo; h < hi; h += HB) {
#pragma unroll
                for (int j = 0; j < HB; ++j)
#pragma unroll
                    for (int i = 0; i < (kBack ? 4 : 2); ++i) these[j][i] = next[j][i];
                ask(h + HB);
                float r[HB];
                float2 x[HB][4];
#pragma unroll
                for (int j = 0; j < HB; ++j) {
                    float2 v[2];
                    these[j][0].get(v);
                    x[j][0] = v[0]; x[j][1] = v[1];
                    these[j][1].get(v);
                    x[j][2] = v[0]; x[j][3] = v[1];
                    if (!on || h + j >= hi) x[j][0] = x[j][1] = x[j][2] = x[j][3] = both(0.f);
                    float2 ss = mul2(x[j][0], x[j][0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) ss = fma2(x[j][i], x[j][i], ss);
                    r[j] = ss.x + ss.y;
                }
#pragma unroll
                for (int j = 0; j < HB; ++j) {
                    r[j] = rsqrtf(fmaf(group_sum(r[j]), per, A.eps));
                    if (kBack && h + j >= hi) r[j] = 0.f;      // no head: without an eps its zeros would be made NaN and counted in the sums
                }
                if constexpr (!kBack) {
#pragma unroll
                    for (int j = 0; j < HB; ++j) {
                        if (s < 2) {      // (values go into the cache as they are)
                            float2 h0[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) h0[i] = mul2(mul2(x[j][i], both(r[j])), w[i]);
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                x[j][i] = fma2(h0[i], cosine[i], neg2(mul2(h0[2 + i], sine[i])));
                                x[j][2 + i] = fma2(h0[2 + i], cosine[i], mul2(h0[i], sine[i]));
                            }
                        }
                        if (writes && h + j < hi) {
                            store4(py, x[j][0], x[j][1]);
                            store4(py + other, x[j][2], x[j][3]);
                        }
                        py += S.y.head;
                    }
                } else {
                    float dot[HB];
                    float2 um[HB][4];
#pragma unroll
                    for (int j = 0; j < HB; ++j) {
                        float2 g[4], v[2], d = both(0.f);
                        these[j][2].get(v);
                        g[0] = v[0]; g[1] = v[1];
                        these[j][3].get(v);
                        g[2] = v[0]; g[3] = v[1];
                        const bool have = on && h + j < hi;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            um[j][i] = fma2(g[i], cosine[i], mul2(g[2 + i], sine[i]));
                            um[j][2 + i] = fma2(g[2 + i], cosine[i], neg2(mul2(g[i], sine[i])));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (!have) um[j][i] = both(0.f);
                            x[j][i] = mul2(x[j][i], both(r[j]));
                            sum[s][i] = fma2(um[j][i], x[j][i], sum[s][i]);
                            um[j][i] = mul2(um[j][i], w[i]);
                            d = fma2(um[j][i], x[j][i], d);
                        }
                        dot[j] = d.x + d.y;
                    }
#pragma unroll
                    for (int j = 0; j < HB; ++j) dot[j] = -group_sum(dot[j]) * per;
#pragma unroll
                    for (int j = 0; j < HB; ++j) {
                        if (writes && h + j < hi) {
                            float2 o[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[i] = mul2(fma2(x[j][i], both(dot[j]), um[j][i]), both(r[j]));
                            store4(py, o[0], o[1]);
                            store4(py + other, o[2], o[3]);
                        }
                        py += S.y.head;
                    }
                }
            }
        }
    }
    if constexpr (kBack) {
        if (!A.part) return;
        // over the groups of the CTA, in their order
        __shared__ float joined[kGroups * 8 * LANES];
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
            if (on) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    joined[group * 8 * LANES + ca + i] = i & 1 ? sum[s][i / 2].y : sum[s][i / 2].x;
                    joined[group * 8 * LANES + cb + i] = i & 1 ? sum[s][2 + i / 2].y : sum[s][2 + i / 2].x;
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < A.dim; c += kThreads) {
                float v = 0.f;
                for (int q = 0; q < kGroups; ++q) v += joined[q * 8 * LANES + c];
                A.part[((int64_t)blockIdx.x * 2 + s) * A.dim + c] = v;
            }
        }
    }
}

// Any head size, alignment and number of pairs: a warp per head, columns lane, lane + 32, ..; a turned
// column reads its partner as well.
template <typename T, bool kBack> __global__ void __launch_bounds__(kThreads) rotary_any_kernel(const __grid_constant__ RotaryArgs A) {
    stream_order();
    constexpr int kCols = kMostDim / 32, kWarps = kThreads / 32;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, total = A.side[0].heads + A.side[1].heads + A.side[2].heads, n = A.pairs;
    const int64_t units = A.batch * A.tokens * A.chunks;
    uint64_t freq[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const int c = lane + 32 * i;
        freq[i] = c < 2 * n ? turn_of(A.frequency[c < n ? c : c - n]) : 0;
    }
    float sum[2][kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) sum[0][i] = sum[1][i] = 0.f;
    for (int64_t u = (int64_t)blockIdx.x * kWarps + warp; u < units; u += (int64_t)gridDim.x * kWarps) {
        const Unit U = unit_at(A, u, total);
        float2 turn[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const int c = lane + 32 * i;
            turn[i] = c < 2 * n ? turned(freq[i], U.pos) : make_float2(0.f, 1.f);
            if (c < n) turn[i].x = -turn[i].x;      // y_c = h_c cos + h_partner * (-sin or sin)
        }
        for (int hh = U.first; hh < U.last; ++hh) {
            const int s = hh < A.side[0].heads ? 0 : hh < A.side[0].heads + A.side[1].heads ? 1 : 2;
            const int h = hh - (s > 0 ? A.side[0].heads : 0) - (s > 1 ? A.side[1].heads : 0);
            const Side& S = A.side[s];
            const T* p = static_cast<const T*>(S.x.p) + U.b * S.x.batch + U.t * S.x.token + (int64_t)h * S.x.head;
            const T* q = kBack ? static_cast<const T*>(S.g.p) + U.b * S.g.batch + U.t * S.g.token + (int64_t)h * S.g.head : nullptr;
            const T* wp = static_cast<const T*>(S.weight);
            T* y = out_at<T>(A, U, s, h);
            float x[kCols], ss = 0.f;
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                const int c = lane + 32 * i;
                x[i] = c < A.dim ? to_f(p[c]) : 0.f;
                ss += x[i] * x[i];
            }
            const float r = rsqrtf(group_sum(ss, 32) / (float)A.dim + A.eps);
            if constexpr (!kBack) {
                if (!y) continue;
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const int c = lane + 32 * i, o = c < n ? c + n : c - n;
                    if (c >= A.dim) break;
                    float v = x[i];
                    if (s < 2) {
                        v = v * r * (wp ? to_f(wp[c]) : 1.f);
                        if (c < 2 * n) v = v * turn[i].y + to_f(p[o]) * r * (wp ? to_f(wp[o]) : 1.f) * turn[i].x;
                    }
                    y[c] = from_f<T>(v);
                }
            } else {
                float um[kCols], dot = 0.f;
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const int c = lane + 32 * i, o = c < n ? c + n : c - n;
                    um[i] = 0.f;
                    if (c >= A.dim) continue;
                    const float g = c < 2 * n ? to_f(q[c]) * turn[i].y - to_f(q[o]) * turn[i].x : to_f(q[c]);
                    x[i] *= r;
                    if (s == 0) sum[0][i] += g * x[i];
                    else sum[1][i] += g * x[i];
                    um[i] = g * (wp ? to_f(wp[c]) : 1.f);
                    dot += um[i] * x[i];
                }
                dot = group_sum(dot, 32) / (float)A.dim;
                if (!S.y.p) continue;
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    if (lane + 32 * i < A.dim) y[lane + 32 * i] = from_f<T>(r * (um[i] - x[i] * dot));
            }
        }
    }
    if constexpr (kBack) {
        if (!A.part) return;
        __shared__ float joined[kWarps * kMostDim];
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kCols; ++i) joined[warp * kMostDim + lane + 32 * i] = sum[s][i];
            __syncthreads();
            for (int c = threadIdx.x; c < A.dim; c += kThreads) {
                float v = 0.f;
                for (int k = 0; k < kWarps; ++k) v += joined[k * kMostDim + c];
                A.part[((int64_t)blockIdx.x * 2 + s) * A.dim + c] = v;
            }
        }
    }
}

template <typename T, bool kBack> const void* rotary_fn(int lanes) {
    return lanes == 0 ? (const void*)rotary_any_kernel<T, kBack>
         : lanes == 4 ? (const void*)rotary_kernel<T, 4, kBack>
         : lanes == 8 ? (const void*)rotary_kernel<T, 8, kBack>
         : lanes == 16 ? (const void*)rotary_kernel<T, 16, kBack> : (const void*)rotary_kernel<T, 32, kBack>;
}
template <bool kBack> const void* rotary_fn(int dtype, int lanes) {
    return dtype == VQC_F32 ? rotary_fn<float, kBack>(lanes) : dtype == VQC_BF16 ? rotary_fn<__nv_bfloat16, kBack>(lanes) : rotary_fn<__half, kBack>(lanes);
}

bool packs4(int dtype, const Heads& h) { return heads_on(h, elem_size(dtype), 4 * elem_size(dtype)); }

// CTAs of a backward that sums over all tokens: as many as stay on the SMs together (8192 tokens of 40 heads of 128, bfloat16: 54 us; with
// six per SM, which take turns, 60; float32, with 170 registers, has one of the two at a time).
int64_t back_ctas(int64_t units, int groups) { return std::max<int64_t>(1, std::min<int64_t>(ceil_div(units, groups), 2LL * sm_count())); }
// Heads of a token that a group of lanes takes: as many as leave every SM 32 groups, which stay on it together (a token's sines and
// cosines are made once per group; 64 groups: 37 us in the place of 34 for a forward of 8192 tokens, 128: 44).
int heads_at_once(int64_t tokens, int heads) {
    int chunk = heads;
    while (chunk > 1 && tokens * ceil_div(heads, chunk) < 32LL * sm_count()) chunk = (chunk + 1) / 2;
    return chunk;
}

vqc_status run(const char* call, int dtype, RotaryArgs& a, bool back, void* gwq, void* gwk, void* ws, size_t ws_bytes, cudaStream_t s) {
    const int heads = a.side[0].heads + a.side[1].heads + a.side[2].heads;
    bool packs = a.dim % 8 == 0 && a.pairs % 4 == 0;
    for (const Side& d : a.side)
        packs = packs && packs4(dtype, d.x) && (!back || packs4(dtype, d.g)) && packs4(dtype, {d.y.p, d.y.batch, d.y.token, d.y.head}) &&
                aligned_to(d.weight, 4 * elem_size(dtype));
    const int lanes = !packs ? 0 : a.dim <= 32 ? 4 : a.dim <= 64 ? 8 : a.dim <= 128 ? 16 : 32, groups = kThreads / (lanes ? lanes : 32);
    a.chunk = heads_at_once(a.batch * a.tokens, heads);
    a.chunks = (int)ceil_div(heads, a.chunk);
    const int64_t units = a.batch * a.tokens * a.chunks;
    int64_t ctas = ceil_div(units, groups);
    if (back) {
        ctas = back_ctas(units, groups);
        if (gwq || gwk) {
            if (!ws || ws_bytes < (size_t)ctas * 2 * a.dim * 4) return set_error(VQC_ERR_WORKSPACE, std::string(call) + ": workspace too small");
            a.part = static_cast<float*>(ws);
        }
        if (units == 0) ctas = 0;
    }
    if (ctas > 0x7fffffff) return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": too many tokens");
    if (ctas > 0) {
        void* args[] = {&a};
        const cudaError_t e = launch(back ? rotary_fn<true>(dtype, lanes) : rotary_fn<false>(dtype, lanes), dim3((unsigned)ctas), kThreads, args, s);
        if (e != cudaSuccess) return cuda_error(e, "rotary launch");
    }
    if (!back || (!gwq && !gwk)) return VQC_OK;
    // (sum_run's first output is the one that is always there)
    if (!gwq) return sum_run(a.part + a.dim, ctas, a.dim, 2 * a.dim, 0, gwk, nullptr, dtype, s);
    return sum_run(a.part, ctas, a.dim, 2 * a.dim, a.dim, gwq, gwk, dtype, s);
}

Rows dense(void* p, int64_t tokens, int heads, int dim) { return {p, tokens * heads * dim, (int64_t)heads * dim, dim}; }

vqc_status checked(const char* call, int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, const vqc_heads* q,
                   const vqc_heads* k, const void* wq, const void* wk, const double* frequencies, int64_t pairs, double eps) {
    if ((dtype != VQC_F32 && dtype != VQC_BF16 && dtype != VQC_F16) || !sequence_sizes_ok(batch, tokens, heads, groups) || dim < 1 || dim > kMostDim ||
        pairs < 0 || 2 * pairs > dim || (pairs && !frequencies) || !(eps >= 0))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": bad type, size or eps");
    const size_t e = elem_size(dtype);
    if (!heads_ok(q, e) || !heads_ok(k, e) || (batch * tokens > 0 && (!q->data || !k->data)))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL or misaligned operand, or a negative stride");
    if (!aligned_to(wq, e) || !aligned_to(wk, e) || !aligned_to(frequencies, 8))
        return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned weight or frequencies");
    return VQC_OK;
}

RotaryArgs arguments(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, const vqc_heads& q, const vqc_heads& k, const void* wq,
                     const void* wk, const double* frequencies, int64_t pairs, double eps) {
    RotaryArgs a{};
    a.side[0] = {heads_of(q), {}, {}, wq, (int)heads};
    a.side[1] = {heads_of(k), {}, {}, wk, (int)groups};
    a.frequency = frequencies;
    a.batch = batch; a.tokens = tokens;
    a.dim = (int)dim; a.pairs = (int)pairs;
    a.eps = (float)eps;
    return a;
}

}  // namespace

bool sequence_sizes_ok(int64_t batch, int64_t tokens, int64_t heads, int64_t groups) {
    return batch >= 0 && tokens >= 0 && batch <= kMostTokens && tokens <= kMostTokens && batch * tokens <= kMostTokens && heads >= 1 &&
           heads <= kMostHeads && groups >= 1 && groups <= kMostHeads;
}

}  // namespace layers
}  // namespace vqc

using namespace vqc;
using namespace vqc::layers;

extern "C" {

vqc_status vqc_norm_rotary_forward(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, const vqc_heads* q,
                                   const vqc_heads* k, const void* weight_q, const void* weight_k, const double* frequencies, int64_t pairs,
                                   const int32_t* positions, int64_t positions_stride, double eps, void* q_out, void* k_out, void* stream) {
    try {
        const char* call = "vqc_norm_rotary_forward";
        const vqc_status st = checked(call, dtype, batch, tokens, heads, groups, dim, q, k, weight_q, weight_k, frequencies, pairs, eps);
        if (st != VQC_OK) return st;
        if ((batch * tokens > 0 && (!q_out || !k_out)) || positions_stride < 0)
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL output or negative stride");
        if (!aligned_to(q_out, 16) || !aligned_to(k_out, 16) || !aligned_to(positions, 4))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned output or positions");
        RotaryArgs a = arguments(batch, tokens, heads, groups, dim, *q, *k, weight_q, weight_k, frequencies, pairs, eps);
        a.position = positions;
        a.position_stride = positions_stride;
        a.side[0].y = dense(q_out, tokens, (int)heads, (int)dim);
        a.side[1].y = dense(k_out, tokens, (int)groups, (int)dim);
        return run(call, dtype, a, false, nullptr, nullptr, nullptr, 0, static_cast<cudaStream_t>(stream));
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

size_t vqc_norm_rotary_workspace_bytes(int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim) {
    if (!sequence_sizes_ok(batch, tokens, heads, groups) || dim < 1 || dim > kMostDim) return (size_t)-1;
    const int chunk = heads_at_once(batch * tokens, (int)(heads + groups));
    // (the fewest groups of lanes of a CTA)
    return align256((size_t)back_ctas(batch * tokens * ceil_div(heads + groups, chunk), kThreads / 32) * 2 * dim * 4);
}

vqc_status vqc_norm_rotary_backward(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim,
                                    const vqc_heads* grad_q_out, const vqc_heads* grad_k_out, const vqc_heads* q, const vqc_heads* k,
                                    const void* weight_q, const void* weight_k, const double* frequencies, int64_t pairs, const int32_t* positions,
                                    int64_t positions_stride, double eps, void* grad_q, void* grad_k, void* grad_weight_q, void* grad_weight_k,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const char* call = "vqc_norm_rotary_backward";
        const vqc_status st = checked(call, dtype, batch, tokens, heads, groups, dim, q, k, weight_q, weight_k, frequencies, pairs, eps);
        if (st != VQC_OK) return st;
        const size_t e = elem_size(dtype);
        if (!heads_ok(grad_q_out, e) || !heads_ok(grad_k_out, e) || (batch * tokens > 0 && (!grad_q_out->data || !grad_k_out->data)) ||
            positions_stride < 0 || !grad_q != !grad_k)
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL or misaligned gradient, a negative stride, or one of two gradients is NULL");
        if (!aligned_to(grad_q, 16) || !aligned_to(grad_k, 16) || !aligned_to(grad_weight_q, e) || !aligned_to(grad_weight_k, e) ||
            !aligned_to(positions, 4) || !aligned_to(workspace, 256))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned output, positions or workspace");
        if (!grad_q && !grad_weight_q && !grad_weight_k) return VQC_OK;
        RotaryArgs a = arguments(batch, tokens, heads, groups, dim, *q, *k, weight_q, weight_k, frequencies, pairs, eps);
        a.position = positions;
        a.position_stride = positions_stride;
        a.side[0].g = heads_of(*grad_q_out);
        a.side[1].g = heads_of(*grad_k_out);
        a.side[0].y = dense(grad_q, tokens, (int)heads, (int)dim);
        a.side[1].y = dense(grad_k, tokens, (int)groups, (int)dim);
        return run(call, dtype, a, true, grad_weight_q, grad_weight_k, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_norm_rotary_step(vqc_real dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t capacity,
                                const vqc_heads* q, const vqc_heads* k, const vqc_heads* v, const void* weight_q, const void* weight_k,
                                const double* frequencies, int64_t pairs, double eps, const int32_t* lengths, void* q_out, const vqc_heads* cache_k,
                                const vqc_heads* cache_v, void* stream) {
    try {
        const char* call = "vqc_norm_rotary_step";
        const vqc_status st = checked(call, dtype, batch, tokens, heads, groups, dim, q, k, weight_q, weight_k, frequencies, pairs, eps);
        if (st != VQC_OK) return st;
        const size_t e = elem_size(dtype);
        if (!heads_ok(v, e) || !heads_ok(cache_k, e) || !heads_ok(cache_v, e) || capacity < 0 || capacity > kMostTokens ||
            (batch * tokens > 0 && (!q_out || !lengths || !v->data || (capacity > 0 && (!cache_k->data || !cache_v->data)))))
            return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": NULL or misaligned operand, output or cache, or a negative stride");
        if (!aligned_to(q_out, 16) || !aligned_to(lengths, 4)) return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": misaligned output or lengths");
        RotaryArgs a = arguments(batch, tokens, heads, groups, dim, *q, *k, weight_q, weight_k, frequencies, pairs, eps);
        a.lengths = lengths;
        a.capacity = capacity;
        a.side[0].y = dense(q_out, tokens, (int)heads, (int)dim);
        a.side[1].y = {const_cast<void*>(cache_k->data), cache_k->batch_stride, cache_k->token_stride, cache_k->head_stride};
        a.side[2] = {heads_of(*v), {}, {const_cast<void*>(cache_v->data), cache_v->batch_stride, cache_v->token_stride, cache_v->head_stride}, nullptr, (int)groups};
        return run(call, dtype, a, false, nullptr, nullptr, nullptr, 0, static_cast<cudaStream_t>(stream));
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

}  // extern "C"
