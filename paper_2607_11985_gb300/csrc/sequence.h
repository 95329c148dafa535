// sequence.h -- the operators of a sequence (head norms with rotation, attention): what their
// translation units share on the host.
#pragma once

#include "layers.h"

namespace vqc {
namespace layers {

// [batch, tokens, heads, dim] with adjacent elements of a head, strides in elements
struct Heads {
    const void* p;
    int64_t batch, token, head;
};
struct Rows {       // the same, written
    void* p;
    int64_t batch, token, head;
};

inline bool heads_ok(const vqc_heads* h, size_t elem) {
    return h && aligned_to(h->data, elem) && h->batch_stride >= 0 && h->token_stride >= 0 && h->head_stride >= 0;
}
inline Heads heads_of(const vqc_heads& h) { return {h.data, h.batch_stride, h.token_stride, h.head_stride}; }
// heads on boundaries of `bytes` bytes
inline bool heads_on(const Heads& h, size_t elem, size_t bytes) {
    const int64_t n = (int64_t)(bytes / elem);
    return aligned_to(h.p, bytes) && h.batch % n == 0 && h.token % n == 0 && h.head % n == 0;
}

constexpr int64_t kMostTokens = (1 << 30) - 1, kMostHeads = 1 << 16;
// batch, tokens and their product, heads and groups within range
bool sequence_sizes_ok(int64_t batch, int64_t tokens, int64_t heads, int64_t groups);

}  // namespace layers
}  // namespace vqc
