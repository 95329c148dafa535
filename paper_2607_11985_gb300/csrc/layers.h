// layers.h -- the classical operators around a circuit (layer norm, linear,
// gated product): what their translation units share on the host.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>
#include <string>

#include "vqc.h"

namespace vqc {

vqc_status set_error(vqc_status s, const std::string& msg);
bool programmatic_launches();   // false where the environment sets VQC_PDL=0

namespace layers {

inline size_t elem_size(int dtype) { return dtype == VQC_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t b) { return (b + 255) & ~size_t(255); }
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

vqc_status cuda_error(cudaError_t e, const char* what);

// A launch that may begin while the kernel before it in the stream ends: its CTAs are
// placed and set up, then wait in stream_order() (layers_elem.cuh), which every kernel
// here calls before it touches memory.  Between two dependent kernels this takes
// away about 2 us.  (In plain stream order where programmatic launches are switched off.)
// The limit of a kernel's dynamic shared memory is raised at its first launch on a device.
cudaError_t launch(const void* fn, dim3 grid, int threads, void** args, cudaStream_t s, size_t shared = 0, int cluster = 1);
int sm_count();   // of the current device (the GB300's 152 where there is none)

// A matrix operand of a product: element (i, k) of the outer index i and the
// contracted index k is p[i * ld + k], or p[k * ld + i] where k_outer is set.
// A 16-bit operand may be the sum of two matrices, the second `second` elements behind
// the first (0: there is none).
struct Operand {
    const void* p;
    int64_t ld;
    bool k_outer;
    int64_t second;
};

enum Form {
    PLAIN = 0,   // y0 = finish(a0 b0^T)
    SUM = 1,     // y0 = finish(a0 b0^T + a1 b1^T)
    PAIR = 2,    // y0 = a0 b0^T and y1 = a1 b1^T in one launch
    GATED = 3    // y0 = act(a0 b0^T + bias0) * (a0 b1^T + bias1)
};

// In the place of an activation: times *scale.
constexpr int kActScale = VQC_ACT_SIGMOID + 1;

// What is done with the sums of a product before they are written.
struct Finish {
    const float* scale;    // of kActScale
    const void* bias[2];   // per column, of the operands' type, or NULL
    const void* res;       // added last, of y's type, or NULL
    int64_t ld_res;
    void* y[2];            // dense [m, n]
    float* z[2];           // sums with their bias, dense [m, n], or NULL
    int64_t m, n;
    int32_t act, dtype, out_dtype, gated;
};

// m x n outputs, contraction over k; every matrix of one form has the same sizes.
struct Product {
    int form;
    int64_t m, n, k;
    Operand a[2], b[2];
    Finish f;
};

// Sums of a contraction that was cut, [splits][1 or 2][m][n] (two for GATED and PAIR),
// still to be joined in the order of the cuts and finished.
struct Join {
    Finish f;
    const float* part;
    int32_t splits, form;
};
constexpr int kMostJoins = 4;
struct Joins {
    Join j[kMostJoins];
    int count;
};
vqc_status join_run(const Joins& joins, cudaStream_t s);

// Bytes of workspace of each of up to two products that run together (or one of them
// alone).  `aligned`: the operands' addresses are multiples of 16 bytes (their
// strides are looked at).
void products_workspace(const Product* p, int count, bool aligned, size_t* bytes);
// Runs products that do not depend on one another, in as few launches as they
// allow; what is left to be joined is added to `joins`.  ws[i], bytes[i]: the workspace
// of product i, in use until the joins have run.
vqc_status products_run(const Product* p, int count, void* const* ws, const size_t* bytes, Joins& joins, cudaStream_t s);

// dz = grad_y * act'(z) (gated: dg and du from grad_h, g and u) and the column sums.
struct ActGrad {
    const void* gy;          // [rows, n] of gy_dtype, rows ld_gy apart
    int64_t ld_gy;
    const float* z[2];       // dense [rows, n]; z[0] may be NULL without an activation
    void* dz[2];             // of dtype, rows ld_dz apart, or NULL
    int64_t ld_dz;
    int64_t second;          // a second part, what the first leaves of dz, goes this many elements behind it (0: there is none)
    void* sum[2];            // [n] of dtype: column sums, or NULL
    float* scale;            // [2] of float16: dz is stored times scale[0], a power of two, and scale[1] = 1 / scale[0]; or NULL
    int64_t rows, n;
    int32_t act, dtype, gy_dtype, gated;
};
size_t act_grad_workspace(int64_t rows, int64_t n, bool gated, bool scaled);
// Column sums of few blocks of rows are left to `joins`.
vqc_status act_grad_run(const ActGrad& a, void* ws, size_t ws_bytes, Joins& joins, cudaStream_t s);

// out_i[c] = sum over j < count of part[i * second + j * ld + c] for i = 0, 1, in a fixed
// order; either output may be NULL.
vqc_status sum_run(const float* part, int64_t count, int64_t n, int64_t ld, int64_t second, void* out0, void* out1, int dtype,
                   cudaStream_t s);

}  // namespace layers
}  // namespace vqc
