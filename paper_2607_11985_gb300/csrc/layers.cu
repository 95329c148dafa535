// layers.cu -- C entry points of the linear and gated operators: argument
// checks, workspaces and the order of the launches.
#include <algorithm>
#include <initializer_list>

#include "layers.h"
#include "layers_tc.h"

namespace vqc {
namespace layers {
namespace {

constexpr int64_t kMost = (1 << 30) - 1;   // TMA coordinates are 32 bits, tiles and all

vqc_status bad(const char* call, const char* what) {
    return set_error(VQC_ERR_INVALID_ARG, std::string(call) + ": " + what);
}

bool real_ok(int t) { return t == VQC_F32 || t == VQC_BF16 || t == VQC_F16; }
bool types_ok(int dtype, int out_dtype) {
    return real_ok(dtype) && real_ok(out_dtype) && (dtype == out_dtype || dtype == VQC_F32 || out_dtype == VQC_F32);
}
bool act_ok(int a) { return a >= VQC_ACT_NONE && a <= VQC_ACT_SIGMOID; }
bool sizes_ok(int64_t rows, int64_t in, int64_t out) {
    return rows >= 0 && rows <= kMost && in >= 1 && in <= kMost && out >= 1 && out <= kMost;
}
// operands lie on boundaries of their elements, outputs on 16 bytes
bool on(const void* p, size_t a) { return aligned_to(p, a); }

// Space of a backward call: dz (and du), then the column sums, then the products.
// Rounding dz to 16 bits adds its own error to the gradients' (1.4 of one rounding
// together).  Where the products are short of work dz is therefore the sum of two 16-bit
// matrices (16 bits of dz in bfloat16, 22 in float16) and the gradients have the error of their one
// rounding, for 10 us at most.  Both gradients, bfloat16, us with one matrix and with two, by
// operations: 0.4e9 (8192 x 1024 to 12) 26.6 and 29.0; 4.3e9 (1024^3) 14.2 and 18.8, gated (777 x 504
// to 1365) 25.6 and 35.0; 5.7e9 (1024 x 1024 to 1365) 18.4 and 28.5; 8.6e9 (2048 x 1024 to 1024) 18.6 and 26.0;
// 17e9 (4096 x 1024 to 1024) 26.8 and 45.4; 24e9 (gated, 1024 x 1024 to 2816) 32.7 and 53.2; from
// there on the second costs its products, near half of the call.  A third matrix would hold all bits of
// a bfloat16 dz and round one gradient in 1000 the other way, for 7 to 13 us more.
// A float16 dz is stored times a power of two, so that its range does not matter (see act_grad_run).
struct BackSpace {
    int64_t ld_dz, second;
    size_t dz, scale, sums, gx, gw, total;
    bool own_dz;
};

Product product_gx(int dtype, int64_t rows, int64_t in, int64_t out, const void* const* dz, int64_t ld_dz, int64_t second,
                   const void* const* w, int64_t ld_w, bool gated, void* gx) {
    Product p{};
    p.form = gated ? SUM : PLAIN;
    p.m = rows; p.n = in; p.k = out;
    for (int i = 0; i < (gated ? 2 : 1); ++i) {
        p.a[i] = {dz[i], ld_dz, false, second};
        p.b[i] = {w[i], ld_w, true, 0};
    }
    p.f.y[0] = gx;
    p.f.m = rows; p.f.n = in;
    p.f.dtype = p.f.out_dtype = dtype;
    return p;
}

Product product_gw(int dtype, int64_t rows, int64_t in, int64_t out, const void* const* dz, int64_t ld_dz, int64_t second,
                   const void* x, int64_t ld_x, bool gated, void* const* gw) {
    Product p{};
    p.form = gated ? PAIR : PLAIN;
    p.m = out; p.n = in; p.k = rows;
    for (int i = 0; i < (gated ? 2 : 1); ++i) {
        p.a[i] = {dz[i], ld_dz, true, second};
        p.b[i] = {x, ld_x, true, 0};
        p.f.y[i] = gw[i];
    }
    p.f.m = out; p.f.n = in;
    p.f.dtype = p.f.out_dtype = dtype;
    return p;
}

Product product_forward(int dtype, int out_dtype, int64_t rows, int64_t in, int64_t out, const void* x, int64_t ld_x,
                        const void* const* w, int64_t ld_w, int act, bool gated) {
    Product p{};
    p.form = gated ? GATED : PLAIN;
    p.m = rows; p.n = out; p.k = in;
    p.a[0] = {x, ld_x, false, 0};
    for (int i = 0; i < (gated ? 2 : 1); ++i) p.b[i] = {w[i], ld_w, false, 0};
    p.f.m = rows; p.f.n = out;
    p.f.act = act; p.f.dtype = dtype; p.f.out_dtype = out_dtype; p.f.gated = gated;
    return p;
}

BackSpace back_space(int dtype, int out_dtype, int64_t rows, int64_t in, int64_t out, int64_t ld_x, int64_t ld_w,
                     int64_t ld_gy, int act, bool gated, bool aligned) {
    BackSpace b{};
    b.own_dz = gated || act != VQC_ACT_NONE || dtype != out_dtype;
    b.ld_dz = b.own_dz ? (out + 7) / 8 * 8 : ld_gy;
    const bool two = b.own_dz && dtype != VQC_F32 && 4.0 * rows * in * out * (gated ? 2 : 1) <= 6e9;
    b.second = two ? (rows * b.ld_dz + 127) / 128 * 128 : 0;
    b.dz = b.own_dz ? align256((size_t)(two ? 2 * b.second : rows * b.ld_dz) * elem_size(dtype)) : 0;
    b.scale = b.own_dz && dtype == VQC_F16 ? 256 : 0;
    b.sums = act_grad_workspace(rows, out, gated, b.scale > 0);
    const void* none[2] = {nullptr, nullptr};
    void* nothing[2] = {nullptr, nullptr};
    const Product p[2] = {product_gx(dtype, rows, in, out, none, b.ld_dz, b.second, none, ld_w, gated, nullptr),
                          product_gw(dtype, rows, in, out, none, b.ld_dz, b.second, nullptr, ld_x, gated, nothing)};
    size_t bytes[2];
    products_workspace(p, 2, aligned, bytes);
    b.gx = bytes[0];
    b.gw = bytes[1];
    b.total = b.dz * (gated ? 2 : 1) + b.scale + b.sums + b.gx + b.gw;
    return b;
}

vqc_status forward(const char* call, int dtype, int out_dtype, int64_t rows, int64_t in, int64_t out, const void* x,
                   int64_t ld_x, const void* const* w, int64_t ld_w, const void* const* bias, int act, bool gated,
                   const void* res, int64_t ld_res, void* y, float* saved, void* ws, size_t ws_bytes, void* stream) {
    if (!types_ok(dtype, out_dtype)) return bad(call, "bad element types");
    if (!act_ok(act)) return bad(call, "unknown activation");
    if (!sizes_ok(rows, in, out)) return bad(call, "sizes out of range");
    if (ld_x < in || ld_w < in || (res && ld_res < out)) return bad(call, "a stride is smaller than its row");
    if (!w[0] || (gated && !w[1]) || (rows > 0 && (!x || !y))) return bad(call, "NULL operand or output");
    const size_t e = elem_size(dtype), eo = elem_size(out_dtype);
    if (!on(x, e) || !on(w[0], e) || (gated && !on(w[1], e)) || !on(bias[0], e) || (gated && !on(bias[1], e)) ||
        !on(res, eo) || !on(y, 16) || !on(saved, 16) || !on(ws, 256))
        return bad(call, "misaligned operand, output or workspace");
    const vqc_status before = layers_pending();
    if (before != VQC_OK) return before;
    Product p = product_forward(dtype, out_dtype, rows, in, out, x, ld_x, w, ld_w, act, gated);
    p.f.bias[0] = bias[0];
    p.f.bias[1] = gated ? bias[1] : nullptr;
    p.f.res = res;
    p.f.ld_res = ld_res;
    p.f.y[0] = y;
    p.f.z[0] = saved;
    p.f.z[1] = saved && gated ? saved + rows * out : nullptr;
    Joins joins{};
    const vqc_status st = products_run(&p, 1, &ws, &ws_bytes, joins, static_cast<cudaStream_t>(stream));
    return st == VQC_OK ? join_run(joins, static_cast<cudaStream_t>(stream)) : st;
}

vqc_status backward(const char* call, int dtype, int out_dtype, int64_t rows, int64_t in, int64_t out, const void* gy,
                    int64_t ld_gy, const void* x, int64_t ld_x, const void* const* w, int64_t ld_w, const float* saved,
                    int act, bool gated, void* gx, void* const* gw, void* const* gb, void* ws, size_t ws_bytes,
                    void* stream) {
    if (!types_ok(dtype, out_dtype)) return bad(call, "bad element types");
    if (!act_ok(act)) return bad(call, "unknown activation");
    if (!sizes_ok(rows, in, out)) return bad(call, "sizes out of range");
    if (ld_x < in || ld_w < in || ld_gy < out) return bad(call, "a stride is smaller than its row");
    if (rows > 0 && (!gy || (!saved && (gated || act != VQC_ACT_NONE)))) return bad(call, "NULL grad or saved values");
    if ((gw[0] && rows > 0 && !x) || (gx && (!w[0] || (gated && !w[1])))) return bad(call, "NULL operand");
    if (gated && (!gw[0] != !gw[1] || !gb[0] != !gb[1])) return bad(call, "one of two gradients is NULL");
    const size_t e = elem_size(dtype), eo = elem_size(out_dtype);
    if (!on(gy, eo) || !on(x, e) || !on(w[0], e) || (gated && !on(w[1], e)) || !on(saved, 4) || !on(gx, 16) ||
        !on(gw[0], 16) || (gated && !on(gw[1], 16)) || !on(gb[0], 16) || (gated && !on(gb[1], 16)) || !on(ws, 256))
        return bad(call, "misaligned operand, output or workspace");
    const vqc_status before = layers_pending();
    if (before != VQC_OK) return before;
    const bool aligned = on(x, 16) && on(w[0], 16) && (!gated || on(w[1], 16)) && on(gy, 16);
    const BackSpace b = back_space(dtype, out_dtype, rows, in, out, ld_x, ld_w, ld_gy, act, gated, aligned);
    if (ws_bytes < b.total || !ws) return set_error(VQC_ERR_WORKSPACE, std::string(call) + ": workspace too small");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* at = static_cast<char*>(ws);
    Joins joins{};
    const bool need_dz = (gx || gw[0]) && b.own_dz;
    const void* dz[2] = {gy, nullptr};
    ActGrad g{};
    if (need_dz) {
        for (int i = 0; i < (gated ? 2 : 1); ++i) { g.dz[i] = at + i * b.dz; dz[i] = g.dz[i]; }
    }
    at += b.dz * (gated ? 2 : 1);
    if (need_dz && b.scale && rows > 0) g.scale = reinterpret_cast<float*>(at);
    at += b.scale;
    if (need_dz || gb[0]) {
        g.gy = gy; g.ld_gy = ld_gy;
        g.z[0] = saved; g.z[1] = gated ? saved + rows * out : nullptr;
        g.ld_dz = b.ld_dz;
        g.second = b.second;
        g.sum[0] = gb[0]; g.sum[1] = gated ? gb[1] : nullptr;
        g.rows = rows; g.n = out;
        g.act = act; g.dtype = dtype; g.gy_dtype = out_dtype; g.gated = gated;
        const vqc_status st = act_grad_run(g, at, b.sums, joins, s);
        if (st != VQC_OK) return st;
    }
    at += b.sums;
    Product p[2];
    void* spaces[2];
    size_t bytes[2];
    int count = 0;
    if (gx) {
        p[count] = product_gx(dtype, rows, in, out, dz, b.ld_dz, b.second, w, ld_w, gated, gx);
        if (g.scale) {
            p[count].f.scale = g.scale + 1;
            p[count].f.act = kActScale;
        }
        spaces[count] = at;
        bytes[count++] = b.gx;
    }
    if (gw[0]) {
        p[count] = product_gw(dtype, rows, in, out, dz, b.ld_dz, b.second, x, ld_x, gated, gw);
        if (g.scale) {
            p[count].f.scale = g.scale + 1;
            p[count].f.act = kActScale;
        }
        spaces[count] = at + b.gx;
        bytes[count++] = b.gw;
    }
    const vqc_status st = products_run(p, count, spaces, bytes, joins, s);
    return st == VQC_OK ? join_run(joins, s) : st;
}

size_t workspace(int mode, int dtype, int out_dtype, int64_t rows, int64_t in, int64_t out, int64_t ld_x, int64_t ld_w,
                 int64_t ld_gy, int act, bool gated, int aligned) {
    if ((mode != 0 && mode != 1) || !types_ok(dtype, out_dtype) || !act_ok(act) || !sizes_ok(rows, in, out) ||
        ld_x < in || ld_w < in || (mode == 1 && ld_gy < out))
        return (size_t)-1;
    if (mode == 1) return back_space(dtype, out_dtype, rows, in, out, ld_x, ld_w, ld_gy, act, gated, aligned != 0).total;
    const void* none[2] = {nullptr, nullptr};
    const Product p = product_forward(dtype, out_dtype, rows, in, out, nullptr, ld_x, none, ld_w, act, gated);
    size_t bytes = 0;
    products_workspace(&p, 1, aligned != 0, &bytes);
    return bytes;
}

}  // namespace
}  // namespace layers
}  // namespace vqc

using namespace vqc;

extern "C" {

vqc_status vqc_linear_forward(vqc_real dtype, vqc_real out_dtype, int64_t rows, int64_t in, int64_t out, const void* x,
                              int64_t x_stride, const void* weight, int64_t weight_stride, const void* bias,
                              vqc_activation act, const void* residual, int64_t residual_stride, void* y, float* saved,
                              void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const void* w[2] = {weight, nullptr};
        const void* b[2] = {bias, nullptr};
        return layers::forward("vqc_linear_forward", dtype, out_dtype, rows, in, out, x, x_stride, w, weight_stride, b, act,
                               false, residual, residual_stride, y, saved, workspace, workspace_bytes, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_linear_backward(vqc_real dtype, vqc_real out_dtype, int64_t rows, int64_t in, int64_t out,
                               const void* grad_y, int64_t grad_y_stride, const void* x, int64_t x_stride,
                               const void* weight, int64_t weight_stride, const float* saved, vqc_activation act,
                               void* grad_x, void* grad_weight, void* grad_bias, void* workspace, size_t workspace_bytes,
                               void* stream) {
    try {
        const void* w[2] = {weight, nullptr};
        void* gw[2] = {grad_weight, nullptr};
        void* gb[2] = {grad_bias, nullptr};
        return layers::backward("vqc_linear_backward", dtype, out_dtype, rows, in, out, grad_y, grad_y_stride, x, x_stride,
                                w, weight_stride, saved, act, false, grad_x, gw, gb, workspace, workspace_bytes, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_gated_forward(vqc_real dtype, int64_t rows, int64_t in, int64_t out, const void* x, int64_t x_stride,
                             const void* weight_gate, const void* weight_up, int64_t weight_stride,
                             const void* bias_gate, const void* bias_up, vqc_activation act, void* h, float* saved,
                             void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const void* w[2] = {weight_gate, weight_up};
        const void* b[2] = {bias_gate, bias_up};
        return layers::forward("vqc_gated_forward", dtype, dtype, rows, in, out, x, x_stride, w, weight_stride, b, act, true,
                               nullptr, 0, h, saved, workspace, workspace_bytes, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

vqc_status vqc_gated_backward(vqc_real dtype, int64_t rows, int64_t in, int64_t out, const void* grad_h,
                              int64_t grad_h_stride, const void* x, int64_t x_stride, const void* weight_gate,
                              const void* weight_up, int64_t weight_stride, const float* saved, vqc_activation act,
                              void* grad_x, void* grad_weight_gate, void* grad_weight_up, void* grad_bias_gate,
                              void* grad_bias_up, void* workspace, size_t workspace_bytes, void* stream) {
    try {
        const void* w[2] = {weight_gate, weight_up};
        void* gw[2] = {grad_weight_gate, grad_weight_up};
        void* gb[2] = {grad_bias_gate, grad_bias_up};
        return layers::backward("vqc_gated_backward", dtype, dtype, rows, in, out, grad_h, grad_h_stride, x, x_stride, w,
                                weight_stride, saved, act, true, grad_x, gw, gb, workspace, workspace_bytes, stream);
    } catch (...) {
        return VQC_ERR_OUT_OF_MEMORY;
    }
}

size_t vqc_linear_workspace_bytes(int32_t mode, vqc_real dtype, vqc_real out_dtype, int64_t rows, int64_t in,
                                  int64_t out, int64_t x_stride, int64_t weight_stride, int64_t grad_y_stride,
                                  vqc_activation act, int32_t aligned) {
    return layers::workspace(mode, dtype, out_dtype, rows, in, out, x_stride, weight_stride, grad_y_stride, act, false,
                             aligned);
}

size_t vqc_gated_workspace_bytes(int32_t mode, vqc_real dtype, int64_t rows, int64_t in, int64_t out, int64_t x_stride,
                                 int64_t weight_stride, int32_t aligned) {
    return layers::workspace(mode, dtype, dtype, rows, in, out, x_stride, weight_stride, out, VQC_ACT_SILU, true, aligned);
}

}  // extern "C"
