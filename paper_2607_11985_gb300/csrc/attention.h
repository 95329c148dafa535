// attention.h -- what the translation units of attention share.
#pragma once

#include "sequence.h"

namespace vqc {
namespace layers {

// Which keys a query sees: j <= i < length and (i - j < window or j < sinks).
struct Sight {
    const int32_t* lengths;      // [batch], or NULL: all tokens
    int64_t tokens, window, sinks;
};

struct AttentionArgs {
    Heads q, k, v, g;            // g: the incoming gradient
    Sight sight;
    void* o;                     // dense [batch, tokens, heads, dim]
    float* saved;                // forward: lse [batch, heads, tokens], or NULL
    const float* lse;            // backward
    float* d;                    // g . o of the rows, [batch, heads, tokens]
    void *gq, *gk, *gv;          // dense
    float* part;                 // FP32 kernels: keys' sums of each head, or NULL
    int64_t batch;
    float scale, scale2;         // scale2: times log2(e)
    int heads, groups, dim, dtype;
};

constexpr int64_t kMostDim = 256;

// On the tensor cores (attention_tc.cu).  `aligned`: q, k, v and the gradient, and their strides, lie on 16 bytes.
bool attention_tc_takes(int dtype, int64_t dim);
size_t attention_tc_workspace(int mode, int dtype, int64_t batch, int64_t tokens, int64_t heads, int64_t groups, int64_t dim, int64_t window, int64_t sinks,
                              bool aligned);
vqc_status attention_tc_backward(const AttentionArgs& a, void* ws, size_t bytes, cudaStream_t s);
vqc_status attention_tc_forward(const AttentionArgs& a, void* ws, size_t bytes, cudaStream_t s);

}  // namespace layers
}  // namespace vqc
