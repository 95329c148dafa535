// layers_torch.cpp -- the layer operators on torch tensors: argument checks, outputs and
// workspaces, the calls of the C ABI, and the autograd functions.
//
// A call on a few rows costs its host path.  Through Python and ctypes a
// forward took 12-20 us and a backward 22-35 us on the GB300's host (allocations
// 1.7 us each, argument conversion, checks), and under autograd, whose backward runs on
// a thread of its own, four times that; so these operators alone of the package
// have their binding in C++.  No kernel is here and no arithmetic.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <cstdint>
#include <optional>
#include <stdexcept>
#include <string>

#include "vqc.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Function;
using torch::autograd::variable_list;

// an argument that Python reports as ValueError
struct Refused : std::invalid_argument {
    using std::invalid_argument::invalid_argument;
};
// a status of the C ABI, reported as binding.VQCError
struct Status : std::runtime_error {
    vqc_status status;
    explicit Status(vqc_status s) : std::runtime_error(vqc_last_error()), status(s) {}
};
void check(vqc_status s) {
    if (s != VQC_OK) throw Status(s);
}

int code_of(at::ScalarType t) {
    return t == at::kFloat ? VQC_F32 : t == at::kBFloat16 ? VQC_BF16 : t == at::kHalf ? VQC_F16 : -1;
}
at::ScalarType type_of(int64_t code) { return code == VQC_F32 ? at::kFloat : code == VQC_BF16 ? at::kBFloat16 : at::kHalf; }

std::string told(const Tensor& t) {
    if (!t.defined()) return "None";
    std::string s = std::string(c10::toString(t.scalar_type())) + " on " + t.device().str() + " [";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

bool here(const Tensor& t) { return t.is_cuda() && t.get_device() == c10::cuda::current_device(); }

// A view that torch negates when it reads it, so read.  (Asking torch to resolve it is a call through the
// dispatcher, 0.7 us a tensor: only where it is one.)
Tensor as_read(const Tensor& t) { return t.is_neg() ? t.resolve_neg() : t; }

// Every operand comes by here: a tangent, which no operator carries on, is refused, not dropped.
void no_tangent(const Tensor& t, const char* name) {
    if (t._fw_grad(0).defined())
        throw std::runtime_error(std::string("forward-mode derivatives of the layer operators are not implemented (") + name + " has a tangent)");
}

// [rows, cols] with adjacent row elements, `ld` elements from row to row
struct Matrix {
    Tensor t;
    int64_t rows, cols, ld;
    int code;
    void* data() const { return t.data_ptr(); }
};
Matrix matrix(const Tensor& given, const char* name) {
    const int code = given.defined() ? code_of(given.scalar_type()) : -1;
    if (code < 0 || given.dim() == 0 || !here(given))
        throw Refused(std::string(name) + " must be a CUDA float32, bfloat16 or float16 tensor on the current device (got " + told(given) + ")");
    const int64_t cols = given.size(given.dim() - 1);
    if (cols < 1) throw Refused(std::string(name) + " must have at least one column (got " + told(given) + ")");
    no_tangent(given, name);
    Matrix m{as_read(given), 0, cols, cols, code};
    if (given.dim() != 2) m.t = m.t.reshape({-1, cols});
    m.rows = m.t.size(0);
    if (m.t.is_contiguous()) return m;
    const int64_t ld = m.t.stride(0);
    if ((m.t.stride(1) != 1 && cols > 1) || (ld < cols && m.rows > 1)) m.t = m.t.contiguous();
    else m.ld = std::max(ld, cols);
    return m;
}
Matrix like(const Tensor& given, int64_t rows, int64_t cols, int code, const char* name) {
    Matrix m = matrix(given, name);
    if ((rows >= 0 && m.rows != rows) || m.cols != cols || m.code != code)
        throw Refused(std::string(name) + " must have " + (rows >= 0 ? std::to_string(rows) + " " : "") + "rows of " + std::to_string(cols) +
                      " elements of " + c10::toString(type_of(code)) + " (got " + told(given) + ")");
    return m;
}
Matrix weight(const Tensor& given, int64_t cols, int code, const char* name) {
    if (!given.defined() || given.dim() != 2 || given.size(0) < 1)
        throw Refused(std::string(name) + " must have two axes (got " + told(given) + ")");
    return like(given, -1, cols, code, name);
}
Tensor vector(const Tensor& given, int64_t n, int code, const char* name) {
    if (!given.defined()) return given;
    if (given.scalar_type() != type_of(code) || given.dim() != 1 || given.size(0) != n || !here(given))
        throw Refused(std::string(name) + " must be a CUDA " + c10::toString(type_of(code)) + " tensor of " + std::to_string(n) +
                      " elements on the current device (got " + told(given) + ")");
    no_tangent(given, name);
    return as_read(given).contiguous();
}
const float* saved_of(const Tensor& t, at::IntArrayRef shape) {
    if (!t.defined() || t.is_neg() || t.sizes() != shape || t.scalar_type() != at::kFloat || !t.is_contiguous() || !here(t))
        throw Refused("saved must be what the forward returned for these rows, on the current device (got " + told(t) + ")");
    no_tangent(t, "saved");
    return static_cast<const float*>(t.data_ptr());
}
void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
bool aligned(std::initializer_list<const void*> p) {
    uintptr_t any = 0;
    for (const void* q : p) any |= reinterpret_cast<uintptr_t>(q);
    return (any & 15) == 0;
}
// x's leading axes with `cols` columns
Tensor output(const Tensor& x, int64_t cols, at::ScalarType type) {
    auto shape = x.sizes().vec();
    shape.back() = cols;
    return at::empty(shape, x.options().dtype(type));
}
Tensor fresh(bool wanted, at::IntArrayRef shape, const Tensor& x) { return wanted ? at::empty(shape, x.options()) : Tensor(); }
// A workspace of its own for every call: calls of several threads and streams never share one.
Tensor space(size_t bytes, const Tensor& x) {
    if (bytes == (size_t)-1) throw Refused("sizes out of range");
    return bytes ? at::empty({(int64_t)bytes}, x.options().dtype(at::kByte)) : Tensor();
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// ---------------------------------------------------------------- the calls

std::pair<Tensor, Tensor> norm_forward(const Tensor& x, const Tensor& w, const Tensor& b, double eps, bool save) {
    const Matrix m = matrix(x, "x");
    const Tensor wv = vector(w, m.cols, m.code, "weight"), bv = vector(b, m.cols, m.code, "bias");
    Tensor y = output(x, m.cols, x.scalar_type()), stats;
    if (save) stats = at::empty({m.rows, 2}, x.options().dtype(at::kFloat));
    check(vqc_layer_norm_forward((vqc_real)m.code, m.rows, m.cols, m.data(), m.ld, address(wv), address(bv), eps, y.data_ptr(),
                                 static_cast<float*>(address(stats)), stream()));
    return {y, stats};
}

variable_list norm_backward(const Tensor& gy, const Tensor& x, const Tensor& w, const Tensor& saved, bool need_x, bool need_w, bool need_b) {
    const Matrix m = matrix(x, "x"), g = like(gy, m.rows, m.cols, m.code, "grad_y");
    const Tensor wv = vector(w, m.cols, m.code, "weight");
    const float* stats = saved_of(saved, {m.rows, 2});
    Tensor gx = need_x ? output(x, m.cols, x.scalar_type()) : Tensor();
    Tensor gw = fresh(need_w, {m.cols}, x), gb = fresh(need_b, {m.cols}, x);
    const size_t bytes = need_w || need_b ? vqc_layer_norm_workspace_bytes(m.rows, m.cols) : 0;
    const Tensor ws = space(bytes, x);
    check(vqc_layer_norm_backward((vqc_real)m.code, m.rows, m.cols, g.data(), g.ld, m.data(), m.ld, address(wv), stats, address(gx),
                                  address(gw), address(gb), address(ws), bytes, stream()));
    return {gx, gw, gb};
}

// out_code -1: x's type
int out_of(int code, int64_t out_code) {
    if (out_code < 0) return code;
    if (out_code != code && code != VQC_F32 && out_code != VQC_F32)
        throw Refused(std::string("the output of ") + c10::toString(type_of(code)) + " operands must be of their type or float32 (got " +
                      c10::toString(type_of(out_code)) + ")");
    return (int)out_code;
}

std::pair<Tensor, Tensor> linear_forward(const Tensor& x, const Tensor& w, const Tensor& b, int64_t act, const Tensor& res,
                                         int64_t out_code, bool save) {
    const Matrix m = matrix(x, "x"), wm = weight(w, m.cols, m.code, "weight");
    const int64_t out = wm.rows;
    const Tensor bv = vector(b, out, m.code, "bias");
    const int yc = out_of(m.code, out_code);
    Matrix r{};
    if (res.defined()) r = like(res, m.rows, out, yc, "residual");
    const size_t bytes = vqc_linear_workspace_bytes(0, (vqc_real)m.code, (vqc_real)yc, m.rows, m.cols, out, m.ld, wm.ld, 0, (vqc_activation)act,
                                                    aligned({m.data(), wm.data()}));
    const Tensor ws = space(bytes, x);
    Tensor y = output(x, out, type_of(yc)), z;
    if (save && act != VQC_ACT_NONE) z = at::empty({m.rows, out}, x.options().dtype(at::kFloat));
    check(vqc_linear_forward((vqc_real)m.code, (vqc_real)yc, m.rows, m.cols, out, m.data(), m.ld, wm.data(), wm.ld, address(bv),
                             (vqc_activation)act, address(r.t), r.ld, y.data_ptr(), static_cast<float*>(address(z)), address(ws), bytes,
                             stream()));
    return {y, z};
}

variable_list linear_backward(const Tensor& gy, const Tensor& x, const Tensor& w, const Tensor& saved, int64_t act, bool need_x,
                              bool need_w, bool need_b) {
    const Matrix m = matrix(x, "x"), wm = weight(w, m.cols, m.code, "weight"), g0 = matrix(gy, "grad_y");
    const int64_t out = wm.rows;
    const int yc = out_of(m.code, g0.code);
    const Matrix g = like(g0.t, m.rows, out, yc, "grad_y");
    const float* z = act != VQC_ACT_NONE ? saved_of(saved, {m.rows, out}) : nullptr;
    Tensor gx = need_x ? output(x, m.cols, x.scalar_type()) : Tensor();
    Tensor gw = fresh(need_w, {out, m.cols}, x), gb = fresh(need_b, {out}, x);
    const size_t bytes = vqc_linear_workspace_bytes(1, (vqc_real)m.code, (vqc_real)yc, m.rows, m.cols, out, m.ld, wm.ld, g.ld,
                                                    (vqc_activation)act, aligned({m.data(), wm.data(), g.data()}));
    const Tensor ws = space(bytes, x);
    check(vqc_linear_backward((vqc_real)m.code, (vqc_real)yc, m.rows, m.cols, out, g.data(), g.ld, m.data(), m.ld, wm.data(), wm.ld, z,
                              (vqc_activation)act, address(gx), address(gw), address(gb), address(ws), bytes, stream()));
    return {gx, gw, gb};
}

std::pair<Matrix, Matrix> weight_pair(const Tensor& wg, const Tensor& wu, int64_t cols, int code) {
    Matrix a = weight(wg, cols, code, "weight_gate"), b = weight(wu, cols, code, "weight_up");
    if (a.rows != b.rows) throw Refused("weight_gate and weight_up must have one shape (got " + told(wg) + " and " + told(wu) + ")");
    if (a.ld != b.ld) {
        a.t = a.t.contiguous();
        b.t = b.t.contiguous();
        a.ld = b.ld = cols;
    }
    return {a, b};
}

std::pair<Tensor, Tensor> gated_forward(const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& bg, const Tensor& bu, int64_t act,
                                        bool save) {
    const Matrix m = matrix(x, "x");
    const auto [g, u] = weight_pair(wg, wu, m.cols, m.code);
    const int64_t out = g.rows;
    const Tensor bgv = vector(bg, out, m.code, "bias_gate"), buv = vector(bu, out, m.code, "bias_up");
    const size_t bytes = vqc_gated_workspace_bytes(0, (vqc_real)m.code, m.rows, m.cols, out, m.ld, g.ld, aligned({m.data(), g.data(), u.data()}));
    const Tensor ws = space(bytes, x);
    Tensor h = output(x, out, x.scalar_type()), z;
    if (save) z = at::empty({2, m.rows, out}, x.options().dtype(at::kFloat));
    check(vqc_gated_forward((vqc_real)m.code, m.rows, m.cols, out, m.data(), m.ld, g.data(), u.data(), g.ld, address(bgv), address(buv),
                            (vqc_activation)act, h.data_ptr(), static_cast<float*>(address(z)), address(ws), bytes, stream()));
    return {h, z};
}

variable_list gated_backward(const Tensor& gh, const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& saved, int64_t act,
                             bool need_x, bool need_w, bool need_b) {
    const Matrix m = matrix(x, "x");
    const auto [g, u] = weight_pair(wg, wu, m.cols, m.code);
    const int64_t out = g.rows;
    const Matrix d = like(gh, m.rows, out, m.code, "grad_h");
    const float* z = saved_of(saved, {2, m.rows, out});
    Tensor gx = need_x ? output(x, m.cols, x.scalar_type()) : Tensor();
    Tensor gwg = fresh(need_w, {out, m.cols}, x), gwu = fresh(need_w, {out, m.cols}, x);
    Tensor gbg = fresh(need_b, {out}, x), gbu = fresh(need_b, {out}, x);
    const size_t bytes = vqc_gated_workspace_bytes(1, (vqc_real)m.code, m.rows, m.cols, out, m.ld, g.ld,
                                                   aligned({m.data(), g.data(), u.data(), d.data()}));
    const Tensor ws = space(bytes, x);
    check(vqc_gated_backward((vqc_real)m.code, m.rows, m.cols, out, d.data(), d.ld, m.data(), m.ld, g.data(), u.data(), g.ld, z,
                             (vqc_activation)act, address(gx), address(gwg), address(gwu), address(gbg), address(gbu), address(ws), bytes,
                             stream()));
    return {gx, gwg, gwu, gbg, gbu};
}

// [batch, tokens, heads, dim] with adjacent elements of a head
struct HeadRows {
    Tensor t;
    int code;
    vqc_heads h;
    int64_t size(int i) const { return t.size(i); }
};
HeadRows head_rows(const Tensor& given, const char* name) {
    const int code = given.defined() ? code_of(given.scalar_type()) : -1;
    if (code < 0 || given.dim() != 4 || !here(given))
        throw Refused(std::string(name) + " must be a CUDA float32, bfloat16 or float16 tensor [batch, tokens, heads, dim] on the current device (got " + told(given) + ")");
    if (given.size(2) < 1 || given.size(3) < 1) throw Refused(std::string(name) + " must have a head of at least one element (got " + told(given) + ")");
    no_tangent(given, name);
    HeadRows r{as_read(given), code, {}};
    if (r.t.stride(3) != 1 && r.t.size(3) > 1) r.t = r.t.contiguous();
    r.h = {r.t.data_ptr(), r.t.stride(0), r.t.stride(1), r.t.stride(2)};
    return r;
}
HeadRows head_rows(const Tensor& given, const HeadRows& like, int64_t heads, const char* name) {
    HeadRows r = head_rows(given, name);
    if (r.code != like.code || r.size(0) != like.size(0) || r.size(1) != like.size(1) || (heads > 0 && r.size(2) != heads) || r.size(3) != like.size(3))
        throw Refused(std::string(name) + " does not fit: " + told(given) + " beside " + told(like.t));
    return r;
}
// Sequences, places and heads of a cache by their strides, the shortest first: (stride, size).
using Axes = std::array<std::pair<int64_t, int64_t>, 3>;
Axes axes_of(const Tensor& t) {
    Axes axes;
    for (int i = 0; i < 3; ++i) axes[i] = {t.stride(i), t.size(i)};
    std::sort(axes.begin(), axes.end());
    return axes;
}
// A cache [batch, capacity, groups, dim], read or written in place.
HeadRows cache_rows(const Tensor& given, const HeadRows& q, int64_t groups, int64_t capacity, bool written, const char* name) {
    if (written && given.defined() && (given.is_neg() || (at::GradMode::is_enabled() && given.requires_grad())))
        throw Refused(std::string(name) + " is written: it must be no view that torch negates, and need no gradient");
    HeadRows r = head_rows(given, name);
    if (r.code != q.code || r.size(0) != q.size(0) || (groups > 0 && r.size(2) != groups) || (capacity >= 0 && r.size(1) != capacity) || r.size(3) != q.size(3))
        throw Refused(std::string(name) + " does not fit: " + told(given) + " beside " + told(q.t));
    if (written) {
        // each stride has to step over all places of the shorter ones
        bool apart = r.t.is_same(given);
        int64_t last = r.size(3) - 1;
        for (const auto& [stride, size] : axes_of(r.t)) {
            if (size < 2) continue;
            apart = apart && stride > last;
            last += (size - 1) * stride;
        }
        if (!apart) throw Refused(std::string(name) + " is written: the elements of a head must be adjacent and no two places one (got " + told(given) + ")");
    }
    return r;
}
// The first and last places of two tensors' elements span memory that they share?
bool shares(const Tensor& a, const Tensor& b) {
    auto span = [](const Tensor& t) {
        int64_t last = 0;
        for (int64_t i = 0; i < t.dim(); ++i) last += (t.size(i) - 1) * t.stride(i);
        const char* p = static_cast<const char*>(t.data_ptr());
        return std::make_pair(p, p + (last + 1) * t.element_size());
    };
    if (!a.numel() || !b.numel()) return false;
    const auto x = span(a), y = span(b);
    return x.first < y.second && y.first < x.second;
}
// Is `rest` the distance of two elements of a cache, as a sum of steps along its axes up to the i-th and within a head?  Where each
// stride steps over all places of the shorter ones, what those reach is less than it: a step or two of an axis can be meant.
bool distance_within(const Axes& axes, int i, int64_t dim, int64_t rest) {
    if (i < 0) return rest < dim && -rest < dim;
    const auto [stride, size] = axes[i];
    if (size < 2) return distance_within(axes, i - 1, dim, rest);
    for (int64_t near = rest / stride, d = near - 1; d <= near + 1; ++d)
        if (d < size && -d < size && distance_within(axes, i - 1, dim, rest - d * stride)) return true;
    return false;
}
// Is a place of one cache one of the other, too?  (Caches as cache_rows takes them to be written; where their strides differ: may
// one be?)
bool caches_meet(const Tensor& a, const Tensor& b) {
    if (!shares(a, b)) return false;
    for (int i = 0; i < 3; ++i)
        if (a.size(i) > 1 && a.stride(i) != b.stride(i)) return true;
    const int64_t bytes = static_cast<const char*>(b.data_ptr()) - static_cast<const char*>(a.data_ptr());
    return bytes % a.element_size() || distance_within(axes_of(a), 2, a.size(3), bytes / a.element_size());
}
// The forms for serving have no gradients: better an error than one that is lost.
void without_gradient(std::initializer_list<const Tensor*> all) {
    if (!at::GradMode::is_enabled()) return;
    for (const Tensor* t : all)
        if (t->defined() && t->requires_grad()) throw Refused("a step has no gradients: call it without recording (torch.no_grad) or on detached tensors");
}
Tensor int_rows(const Tensor& given, int64_t batch, int64_t tokens, const char* name) {      // tokens < 0: [batch]
    if (!given.defined()) return given;
    const bool one = tokens < 0;
    const bool fits = one ? given.dim() == 1 && given.size(0) == batch
                          : (given.dim() == 1 && given.size(0) == tokens) ||
                                (given.dim() == 2 && given.size(1) == tokens && (given.size(0) == batch || given.size(0) == 1));
    if (given.scalar_type() != at::kInt || !here(given) || !fits)
        throw Refused(std::string(name) + " must be a CUDA int32 tensor " + (one ? "[batch]" : "[batch, tokens] or [tokens]") + " on the current device (got " + told(given) + ")");
    return given.contiguous();
}

struct Draw {
    double p;
    uint64_t seed, offset;
    Tensor state;      // in the place of the seed, or undefined
    const uint64_t* words() const { return static_cast<const uint64_t*>(address(state)); }
};
Tensor dropout_run(const Tensor& x, const Draw& d, const Tensor& res, bool back) {
    const Matrix m = matrix(x, back ? "grad_y" : "x");
    if (!(d.p >= 0) || !(d.p < 1)) throw Refused("p must be at least 0 and less than 1 (got " + std::to_string(d.p) + ")");
    if (d.state.defined() && (d.state.scalar_type() != at::kLong || d.state.dim() != 1 || d.state.size(0) != 2 || !d.state.is_contiguous() || !here(d.state)))
        throw Refused("seed must be an integer, or a dense CUDA int64 tensor of two elements (seed, offset) on the current device (got " + told(d.state) + ")");
    Tensor y = output(x, m.cols, x.scalar_type());
    if (back) {
        check(vqc_dropout_backward((vqc_real)m.code, m.rows, m.cols, m.data(), m.ld, d.p, d.seed, d.offset, d.words(), y.data_ptr(), stream()));
        return y;
    }
    Matrix r{};
    if (res.defined()) r = like(res, m.rows, m.cols, m.code, "residual");
    check(vqc_dropout_forward((vqc_real)m.code, m.rows, m.cols, m.data(), m.ld, address(r.t), r.ld, d.p, d.seed, d.offset, d.words(), y.data_ptr(),
                              stream()));
    return y;
}

// What turns and scales queries and keys.
struct Turn {
    Tensor wq, wk, frequencies, positions;
    double eps;
    int64_t pairs() const { return frequencies.defined() ? frequencies.size(0) : 0; }
};
Turn turn_of(const HeadRows& q, const Turn& t) {
    const int64_t dim = q.size(3);
    Turn r{vector(t.wq, dim, q.code, "weight_q"), vector(t.wk, dim, q.code, "weight_k"), t.frequencies, int_rows(t.positions, q.size(0), q.size(1), "positions"), t.eps};
    if (r.frequencies.defined()) {
        if (r.frequencies.scalar_type() != at::kDouble || r.frequencies.dim() != 1 || 2 * r.frequencies.size(0) > dim || !here(r.frequencies))
            throw Refused("frequencies must be a CUDA float64 tensor of at most half as many elements as a head on the current device (got " + told(r.frequencies) + ")");
        no_tangent(r.frequencies, "frequencies");
        r.frequencies = as_read(r.frequencies).contiguous();
    }
    if (!(t.eps >= 0)) throw Refused("eps must not be negative (got " + std::to_string(t.eps) + ")");
    if (dim > 256) throw Refused("heads of at most 256 elements (got " + told(q.t) + ")");
    return r;
}
int64_t rows_apart(const Tensor& positions, const HeadRows& q) {
    return positions.defined() && positions.dim() == 2 && positions.size(0) == q.size(0) ? q.size(1) : 0;
}
Tensor dense(const HeadRows& like, int64_t heads) { return at::empty({like.size(0), like.size(1), heads, like.size(3)}, like.t.options()); }

variable_list rotary_forward(const Tensor& q, const Tensor& k, const Turn& given) {
    const HeadRows a = head_rows(q, "q"), b = head_rows(k, a, -1, "k");
    const Turn t = turn_of(a, given);
    Tensor yq = dense(a, a.size(2)), yk = dense(a, b.size(2));
    check(vqc_norm_rotary_forward((vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), &a.h, &b.h, address(t.wq), address(t.wk),
                                  static_cast<const double*>(address(t.frequencies)), t.pairs(), static_cast<const int32_t*>(address(t.positions)),
                                  rows_apart(t.positions, a), t.eps, yq.data_ptr(), yk.data_ptr(), stream()));
    return {yq, yk};
}
variable_list rotary_backward(const Tensor& gq, const Tensor& gk, const Tensor& q, const Tensor& k, const Turn& given, bool need_x, bool need_wq, bool need_wk) {
    const HeadRows a = head_rows(q, "q"), b = head_rows(k, a, -1, "k");
    const HeadRows ga = head_rows(gq, a, a.size(2), "grad_q"), gb = head_rows(gk, a, b.size(2), "grad_k");
    const Turn t = turn_of(a, given);
    need_wq = need_wq && t.wq.defined();
    need_wk = need_wk && t.wk.defined();
    Tensor xq = need_x ? dense(a, a.size(2)) : Tensor(), xk = need_x ? dense(a, b.size(2)) : Tensor();
    Tensor wq = fresh(need_wq, {a.size(3)}, a.t), wk = fresh(need_wk, {a.size(3)}, a.t);
    const size_t bytes = need_wq || need_wk ? vqc_norm_rotary_workspace_bytes(a.size(0), a.size(1), a.size(2), b.size(2), a.size(3)) : 0;
    const Tensor ws = space(bytes, a.t);
    check(vqc_norm_rotary_backward((vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), &ga.h, &gb.h, &a.h, &b.h, address(t.wq),
                                   address(t.wk), static_cast<const double*>(address(t.frequencies)), t.pairs(),
                                   static_cast<const int32_t*>(address(t.positions)), rows_apart(t.positions, a), t.eps, address(xq), address(xk),
                                   address(wq), address(wk), address(ws), bytes, stream()));
    return {xq, xk, wq, wk};
}
void written(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
Tensor rotary_step(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& ck, const Tensor& cv, const Tensor& lengths, const Turn& given) {
    const HeadRows a = head_rows(q, "q"), b = head_rows(k, a, -1, "k"), c = head_rows(v, a, b.size(2), "v");
    const HeadRows kc = cache_rows(ck, a, b.size(2), -1, true, "cache_k"), vc = cache_rows(cv, a, b.size(2), kc.size(1), true, "cache_v");
    without_gradient({&q, &k, &v, &given.wq, &given.wk, &given.frequencies});
    // (views of one tensor that holds keys and values are fine: other places)
    if (caches_meet(kc.t, vc.t)) throw Refused("cache_k and cache_v are written: no place of one may be one of the other (got " + told(ck) + " and " + told(cv) + ")");
    for (const HeadRows* from : {&a, &b, &c})
        if (shares(from->t, kc.t) || shares(from->t, vc.t)) throw Refused("the caches are written: q, k and v must lie elsewhere");
    const Turn t = turn_of(a, given);
    if (!lengths.defined()) throw Refused("lengths must be given");
    const Tensor n = int_rows(lengths, a.size(0), -1, "lengths");
    Tensor yq = dense(a, a.size(2));
    check(vqc_norm_rotary_step((vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), kc.size(1), &a.h, &b.h, &c.h, address(t.wq),
                               address(t.wk), static_cast<const double*>(address(t.frequencies)), t.pairs(), t.eps,
                               static_cast<const int32_t*>(address(n)), yq.data_ptr(), &kc.h, &vc.h, stream()));
    written(ck);
    written(cv);
    return yq;
}

// What a query sees.
struct Sight {
    int64_t window, sinks;
    double scale;       // 0: 1 / sqrt(dim)
    Tensor lengths;
};
Sight sight_of(const HeadRows& q, int64_t groups, const Sight& s) {
    if (s.window < 0 || s.sinks < 0) throw Refused("window must be None or at least 1, sinks at least 0");
    if (q.size(2) % groups) throw Refused("the heads of q must be a multiple of those of k (got " + std::to_string(q.size(2)) + " and " + std::to_string(groups) + ")");
    if (q.size(3) > 256) throw Refused("heads of at most 256 elements (got " + told(q.t) + ")");
    Sight r{s.window, s.sinks, s.scale == 0 ? 1.0 / std::sqrt((double)q.size(3)) : s.scale, int_rows(s.lengths, q.size(0), -1, "lengths")};
    if (!(r.scale > 1e-30) || !(r.scale < 1e30)) throw Refused("scale must be positive and within float's range (got " + std::to_string(s.scale) + ")");
    return r;
}
bool on16(const HeadRows& r) {
    const int64_t n = r.code == VQC_F32 ? 4 : 8;
    bool on = aligned({r.h.data});
    for (int i = 0; i < 3; ++i) on = on && (r.t.size(i) == 1 || (r.t.stride(i) > 0 && r.t.stride(i) % n == 0));
    return on;
}
std::pair<Tensor, Tensor> attention_forward(const Tensor& q, const Tensor& k, const Tensor& v, const Sight& given, bool save) {
    const HeadRows a = head_rows(q, "q"), b = head_rows(k, a, -1, "k"), c = head_rows(v, a, b.size(2), "v");
    const Sight s = sight_of(a, b.size(2), given);
    Tensor o = dense(a, a.size(2)), saved;
    if (save) saved = at::empty({a.size(0), a.size(2), a.size(1)}, a.t.options().dtype(at::kFloat));
    const size_t bytes = vqc_attention_workspace_bytes(0, (vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), s.window, s.sinks,
                                                       on16(a) && on16(b) && on16(c));
    const Tensor ws = space(bytes, a.t);
    check(vqc_attention_forward((vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), &a.h, &b.h, &c.h, s.window, s.sinks, s.scale,
                                static_cast<const int32_t*>(address(s.lengths)), o.data_ptr(), static_cast<float*>(address(saved)), address(ws), bytes,
                                stream()));
    return {o, saved};
}
variable_list attention_backward(const Tensor& go, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o, const Tensor& saved,
                                 const Sight& given, bool need_q, bool need_kv) {
    const HeadRows a = head_rows(q, "q"), b = head_rows(k, a, -1, "k"), c = head_rows(v, a, b.size(2), "v"), g = head_rows(go, a, a.size(2), "grad_o");
    const HeadRows y = head_rows(o, a, a.size(2), "o");
    const Sight s = sight_of(a, b.size(2), given);
    const float* lse = saved_of(saved, {a.size(0), a.size(2), a.size(1)});
    const Tensor out = y.t.contiguous();
    Tensor gq = need_q ? dense(a, a.size(2)) : Tensor(), gk = need_kv ? dense(a, b.size(2)) : Tensor(), gv = need_kv ? dense(a, b.size(2)) : Tensor();
    const size_t bytes = vqc_attention_workspace_bytes(1, (vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), s.window, s.sinks,
                                                       on16(a) && on16(b) && on16(c) && on16(g));
    const Tensor ws = space(bytes, a.t);
    check(vqc_attention_backward((vqc_real)a.code, a.size(0), a.size(1), a.size(2), b.size(2), a.size(3), &g.h, &a.h, &b.h, &c.h, out.data_ptr(), lse,
                                 s.window, s.sinks, s.scale, static_cast<const int32_t*>(address(s.lengths)), address(gq), address(gk), address(gv),
                                 address(ws), bytes, stream()));
    return {gq, gk, gv};
}
Tensor attention_step(const Tensor& q, const Tensor& ck, const Tensor& cv, const Sight& given) {
    const HeadRows a = head_rows(q, "q"), kc = cache_rows(ck, a, -1, -1, false, "cache_k"), vc = cache_rows(cv, a, kc.size(2), kc.size(1), false, "cache_v");
    if (!given.lengths.defined()) throw Refused("lengths must be given");
    without_gradient({&q, &ck, &cv});
    const Sight s = sight_of(a, kc.size(2), given);
    Tensor o = dense(a, a.size(2));
    const size_t bytes = vqc_attention_step_workspace_bytes(a.size(0), a.size(1), a.size(2), kc.size(2), a.size(3), kc.size(1), s.window, s.sinks);
    const Tensor ws = space(bytes, a.t);
    check(vqc_attention_step((vqc_real)a.code, a.size(0), a.size(1), a.size(2), kc.size(2), a.size(3), kc.size(1), &a.h, &kc.h, &vc.h, s.window, s.sinks,
                             s.scale, static_cast<const int32_t*>(address(s.lengths)), o.data_ptr(), address(ws), bytes, stream()));
    return o;
}

// ---------------------------------------------------------------- autograd

[[noreturn]] variable_list only_once() { throw std::runtime_error("these layer operators can be differentiated once only"); }

// An operand that may be left out enters a function as an optional; the inputs that
// can need a gradient are counted without those left out.
using Optional = std::optional<Tensor>;
Optional optional(const Tensor& t) { return t.defined() ? Optional(t) : Optional(); }
Tensor tensor(const Optional& t) { return t ? *t : Tensor(); }
struct Inputs {
    AutogradContext* ctx;
    int64_t present;     // bit i: input i was given
    int edge = 0;
    bool needed(int i) { return (present >> i & 1) && ctx->needs_input_grad(edge++); }
};

// A function's outputs are tensors all: those that were asked for, put back in their places.
variable_list only(const variable_list& v) {
    variable_list r;
    for (const Tensor& t : v)
        if (t.defined()) r.push_back(t);
    return r;
}
variable_list spread(const variable_list& v, std::initializer_list<bool> asked) {
    variable_list r;
    size_t next = 0;
    for (bool a : asked) r.push_back(a ? v[next++] : Tensor());
    return r;
}

// Under create_graph the gradients are outputs of a function whose own gradient is refused.
struct NormGradients : Function<NormGradients> {
    static variable_list forward(AutogradContext*, const Tensor& gy, const Tensor& x, const Optional& w, const Tensor& saved, bool nx, bool nw, bool nb) {
        return only(norm_backward(gy, x, tensor(w), saved, nx, nw, nb));
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};
struct LinearGradients : Function<LinearGradients> {
    static variable_list forward(AutogradContext*, const Tensor& gy, const Tensor& x, const Tensor& w, const Optional& saved, int64_t act, bool nx,
                                 bool nw, bool nb) {
        return only(linear_backward(gy, x, w, tensor(saved), act, nx, nw, nb));
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};
struct GatedGradients : Function<GatedGradients> {
    static variable_list forward(AutogradContext*, const Tensor& gh, const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& saved,
                                 int64_t act, bool nx, bool nw, bool nb) {
        return only(gated_backward(gh, x, wg, wu, saved, act, nx, nw, nb));
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};

struct NormFunction : Function<NormFunction> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Optional& w, const Optional& b, double eps) {
        auto [y, stats] = norm_forward(x, tensor(w), tensor(b), eps, true);
        if (w) ctx->save_for_backward({x, stats, *w});
        else ctx->save_for_backward({x, stats});
        ctx->saved_data["present"] = (int64_t)(1 | (w ? 2 : 0) | (b ? 4 : 0));
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return variable_list(4);
        const variable_list s = ctx->get_saved_variables();
        const Tensor w = s.size() > 2 ? s[2] : Tensor();
        Inputs in{ctx, ctx->saved_data["present"].toInt()};
        const bool nx = in.needed(0), nw = in.needed(1), nb = in.needed(2);
        variable_list r = at::GradMode::is_enabled() && (nx || nw || nb)
                              ? spread(NormGradients::apply(g[0], s[0], optional(w), s[1], nx, nw, nb), {nx, nw, nb})
                                                     : norm_backward(g[0], s[0], w, s[1], nx, nw, nb);
        r.resize(4);
        return r;
    }
};

struct LinearFunction : Function<LinearFunction> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Optional& b, const Optional& res, int64_t act, int64_t out_code) {
        auto [y, z] = linear_forward(x, w, tensor(b), act, tensor(res), out_code, true);
        if (z.defined()) ctx->save_for_backward({x, w, z});
        else ctx->save_for_backward({x, w});
        ctx->saved_data["present"] = (int64_t)(3 | (b ? 4 : 0) | (res ? 8 : 0));
        ctx->saved_data["act"] = act;
        if (res && res->sizes() != y.sizes()) ctx->saved_data["residual"] = res->sizes().vec();      // as many rows, other leading axes
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return variable_list(6);
        const variable_list s = ctx->get_saved_variables();
        const Tensor z = s.size() > 2 ? s[2] : Tensor();
        const int64_t act = ctx->saved_data["act"].toInt();
        Inputs in{ctx, ctx->saved_data["present"].toInt()};
        const bool nx = in.needed(0), nw = in.needed(1), nb = in.needed(2), nr = in.needed(3);
        variable_list r(3);
        if (nx || nw || nb)
            r = at::GradMode::is_enabled() ? spread(LinearGradients::apply(g[0], s[0], s[1], optional(z), act, nx, nw, nb), {nx, nw, nb})
                                           : linear_backward(g[0], s[0], s[1], z, act, nx, nw, nb);
        const auto shape = ctx->saved_data.find("residual");
        r.push_back(!nr ? Tensor() : shape == ctx->saved_data.end() ? g[0] : g[0].reshape(shape->second.toIntVector()));
        r.resize(6);
        return r;
    }
};

struct GatedFunction : Function<GatedFunction> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& wg, const Tensor& wu, const Optional& bg, const Optional& bu, int64_t act) {
        auto [h, z] = gated_forward(x, wg, wu, tensor(bg), tensor(bu), act, true);
        ctx->save_for_backward({x, wg, wu, z});
        ctx->saved_data["present"] = (int64_t)(7 | (bg ? 8 : 0) | (bu ? 16 : 0));
        ctx->saved_data["act"] = act;
        return h;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return variable_list(6);
        const variable_list s = ctx->get_saved_variables();
        const int64_t act = ctx->saved_data["act"].toInt();
        Inputs in{ctx, ctx->saved_data["present"].toInt()};
        bool need[5];
        for (int i = 0; i < 5; ++i) need[i] = in.needed(i);
        const bool nw = need[1] || need[2], nb = need[3] || need[4];
        variable_list r = at::GradMode::is_enabled() && (need[0] || nw || nb)
                              ? spread(GatedGradients::apply(g[0], s[0], s[1], s[2], s[3], act, need[0], nw, nb), {need[0], nw, nw, nb, nb})
                                                     : gated_backward(g[0], s[0], s[1], s[2], s[3], act, need[0], nw, nb);
        for (int i = 0; i < 5; ++i)
            if (!need[i]) r[i] = Tensor();
        r.resize(6);
        return r;
    }
};

struct DropoutGradient : Function<DropoutGradient> {
    static Tensor forward(AutogradContext*, const Tensor& gy, const Optional& state, double p, int64_t seed, int64_t offset) {
        return dropout_run(gy, {p, (uint64_t)seed, (uint64_t)offset, tensor(state)}, Tensor(), true);
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};
struct RotaryGradients : Function<RotaryGradients> {
    static variable_list forward(AutogradContext*, const Tensor& gq, const Tensor& gk, const Tensor& q, const Tensor& k, const Optional& wq, const Optional& wk,
                                 const Optional& f, const Optional& pos, double eps, bool nx, bool nwq, bool nwk) {
        return only(rotary_backward(gq, gk, q, k, {tensor(wq), tensor(wk), tensor(f), tensor(pos), eps}, nx, nwq, nwk));
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};
struct AttentionGradients : Function<AttentionGradients> {
    static variable_list forward(AutogradContext*, const Tensor& go, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o, const Tensor& saved,
                                 const Optional& lengths, int64_t window, int64_t sinks, double scale, bool nq, bool nkv) {
        return only(attention_backward(go, q, k, v, o, saved, {window, sinks, scale, tensor(lengths)}, nq, nkv));
    }
    static variable_list backward(AutogradContext*, variable_list) { only_once(); }
};

struct DropoutFunction : Function<DropoutFunction> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Optional& res, const Optional& state, double p, int64_t seed, int64_t offset) {
        Tensor y = dropout_run(x, {p, (uint64_t)seed, (uint64_t)offset, tensor(state)}, tensor(res), false);
        if (state) ctx->save_for_backward({*state});      // (a state that has changed since is refused)
        ctx->saved_data["present"] = (int64_t)(1 | (res ? 2 : 0));
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = seed;
        ctx->saved_data["offset"] = offset;
        if (res && res->sizes() != y.sizes()) ctx->saved_data["residual"] = res->sizes().vec();
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return variable_list(6);
        const variable_list s = ctx->get_saved_variables();
        const Tensor state = s.empty() ? Tensor() : s[0];
        Inputs in{ctx, ctx->saved_data["present"].toInt()};
        const bool nx = in.needed(0), nr = in.needed(1);
        const double p = ctx->saved_data["p"].toDouble();
        const int64_t seed = ctx->saved_data["seed"].toInt(), offset = ctx->saved_data["offset"].toInt();
        variable_list r(6);
        if (nx)
            r[0] = at::GradMode::is_enabled() ? DropoutGradient::apply(g[0], optional(state), p, seed, offset)
                                              : dropout_run(g[0], {p, (uint64_t)seed, (uint64_t)offset, state}, Tensor(), true);
        const auto shape = ctx->saved_data.find("residual");
        if (nr) r[1] = shape == ctx->saved_data.end() ? g[0] : g[0].reshape(shape->second.toIntVector());
        return r;
    }
};

struct RotaryFunction : Function<RotaryFunction> {
    static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Optional& wq, const Optional& wk, const Optional& f,
                                 const Optional& pos, double eps) {
        variable_list y = rotary_forward(q, k, {tensor(wq), tensor(wk), tensor(f), tensor(pos), eps});
        variable_list keep = {q, k};
        for (const Optional* t : {&wq, &wk, &f, &pos})
            if (*t) keep.push_back(**t);
        ctx->save_for_backward(keep);
        ctx->saved_data["present"] = (int64_t)(3 | (wq ? 4 : 0) | (wk ? 8 : 0) | (f ? 16 : 0) | (pos ? 32 : 0));
        ctx->saved_data["eps"] = eps;
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined() && !g[1].defined()) return variable_list(7);
        const variable_list s = ctx->get_saved_variables();
        const int64_t present = ctx->saved_data["present"].toInt();
        size_t next = 2;
        auto take = [&](int bit) { return present >> bit & 1 ? s[next++] : Tensor(); };
        Turn t;
        t.wq = take(2);
        t.wk = take(3);
        t.frequencies = take(4);
        t.positions = take(5);
        t.eps = ctx->saved_data["eps"].toDouble();
        Inputs in{ctx, present};
        const bool nq = in.needed(0), nk = in.needed(1), nwq = in.needed(2), nwk = in.needed(3), nx = nq || nk;
        for (int i = 0; i < 2; ++i)      // an output that was not used
            if (!g[i].defined()) g[i] = at::zeros(s[i].sizes(), s[i].options());
        variable_list r(4);
        if (nx || nwq || nwk)
            r = at::GradMode::is_enabled() ? spread(RotaryGradients::apply(g[0], g[1], s[0], s[1], optional(t.wq), optional(t.wk), optional(t.frequencies),
                                                                           optional(t.positions), t.eps, nx, nwq, nwk), {nx, nx, nwq, nwk})
                                           : rotary_backward(g[0], g[1], s[0], s[1], t, nx, nwq, nwk);
        if (!nq) r[0] = Tensor();
        if (!nk) r[1] = Tensor();
        r.resize(7);
        return r;
    }
};

struct AttentionFunction : Function<AttentionFunction> {
    static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const Optional& lengths, int64_t window, int64_t sinks,
                          double scale) {
        auto [o, saved] = attention_forward(q, k, v, {window, sinks, scale, tensor(lengths)}, true);
        if (lengths) ctx->save_for_backward({q, k, v, o, saved, *lengths});
        else ctx->save_for_backward({q, k, v, o, saved});
        ctx->saved_data["window"] = window;
        ctx->saved_data["sinks"] = sinks;
        ctx->saved_data["scale"] = scale;
        return o;
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return variable_list(7);
        const variable_list s = ctx->get_saved_variables();
        const Sight sight{ctx->saved_data["window"].toInt(), ctx->saved_data["sinks"].toInt(), ctx->saved_data["scale"].toDouble(), s.size() > 5 ? s[5] : Tensor()};
        const bool nq = ctx->needs_input_grad(0), nk = ctx->needs_input_grad(1), nv = ctx->needs_input_grad(2), nkv = nk || nv;
        variable_list r(3);
        if (nq || nkv)
            r = at::GradMode::is_enabled() ? spread(AttentionGradients::apply(g[0], s[0], s[1], s[2], s[3], s[4], optional(sight.lengths), sight.window,
                                                                              sight.sinks, sight.scale, nq, nkv), {nq, nkv, nkv})
                                           : attention_backward(g[0], s[0], s[1], s[2], s[3], s[4], sight, nq, nkv);
        if (!nk) r[1] = Tensor();
        if (!nv) r[2] = Tensor();
        r.resize(7);
        return r;
    }
};

bool recorded(std::initializer_list<const Tensor*> inputs) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : inputs)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}
Tensor norm(const Tensor& x, const Tensor& w, const Tensor& b, double eps) {
    return recorded({&x, &w, &b}) ? NormFunction::apply(x, optional(w), optional(b), eps) : norm_forward(x, w, b, eps, false).first;
}
Tensor linear(const Tensor& x, const Tensor& w, const Tensor& b, int64_t act, const Tensor& res, int64_t out_code) {
    return recorded({&x, &w, &b, &res}) ? LinearFunction::apply(x, w, optional(b), optional(res), act, out_code)
                                        : linear_forward(x, w, b, act, res, out_code, false).first;
}
Tensor gated(const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& bg, const Tensor& bu, int64_t act) {
    return recorded({&x, &wg, &wu, &bg, &bu}) ? GatedFunction::apply(x, wg, wu, optional(bg), optional(bu), act)
                                              : gated_forward(x, wg, wu, bg, bu, act, false).first;
}

Tensor dropout(const Tensor& x, const Draw& d, const Tensor& res) {
    return recorded({&x, &res}) ? DropoutFunction::apply(x, optional(res), optional(d.state), d.p, (int64_t)d.seed, (int64_t)d.offset)
                                : dropout_run(x, d, res, false);
}
variable_list rotary(const Tensor& q, const Tensor& k, const Turn& t) {
    if (recorded({&t.frequencies})) throw Refused("frequencies have no gradient: call it without recording (torch.no_grad) or on detached ones");
    return recorded({&q, &k, &t.wq, &t.wk}) ? RotaryFunction::apply(q, k, optional(t.wq), optional(t.wk), optional(t.frequencies), optional(t.positions), t.eps)
                                            : rotary_forward(q, k, t);
}
Tensor attention(const Tensor& q, const Tensor& k, const Tensor& v, const Sight& s) {
    return recorded({&q, &k, &v}) ? AttentionFunction::apply(q, k, v, optional(s.lengths), s.window, s.sinks, s.scale) : attention_forward(q, k, v, s, false).first;
}

// ---------------------------------------------------------------- Python

Tensor tensor_arg(PyObject* o) {
    if (o == Py_None) return Tensor();
    if (!THPVariable_Check(o)) throw Refused(std::string("a tensor was expected (got ") + Py_TYPE(o)->tp_name + ")");
    return THPVariable_Unpack(o);
}
int64_t int_arg(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
double float_arg(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
bool bool_arg(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// The interpreter runs on while the library works (a launch may wait for the GPU's queue).
struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
};
template <typename F> auto released(F f) {
    Released r;
    return f();
}

PyObject* wrapped(const Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* wrapped(const variable_list& v) {
    PyObject* tuple = PyTuple_New((Py_ssize_t)v.size());
    if (!tuple) throw python_error();
    for (size_t i = 0; i < v.size(); ++i) PyTuple_SET_ITEM(tuple, (Py_ssize_t)i, wrapped(v[i]));
    return tuple;
}
PyObject* wrapped(const std::pair<Tensor, Tensor>& p, bool both) {
    return both ? wrapped(variable_list{p.first, p.second}) : wrapped(p.first);
}

template <typename F> PyObject* guarded(Py_ssize_t have, Py_ssize_t want, F f) {
    HANDLE_TH_ERRORS
    if (have != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    } catch (const Status& e) {
        PyObject* binding = PyImport_ImportModule("paper_2607_11985_gb300.binding");
        PyObject* error = binding ? PyObject_GetAttrString(binding, "VQCError") : nullptr;
        PyObject* value = error ? PyObject_CallFunction(error, "is", (int)e.status, e.what()) : nullptr;
        if (value) PyErr_SetObject(error, value);
        Py_XDECREF(value);
        Py_XDECREF(error);
        Py_XDECREF(binding);
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define ARGS PyObject*, PyObject *const *a, Py_ssize_t n

PyObject* py_norm_forward(ARGS) {
    return guarded(n, 5, [&] {
        const Tensor x = tensor_arg(a[0]), w = tensor_arg(a[1]), b = tensor_arg(a[2]);
        const double eps = float_arg(a[3]);
        const bool save = bool_arg(a[4]);
        return wrapped(released([&] { return norm_forward(x, w, b, eps, save); }), save);
    });
}
PyObject* py_norm_backward(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor g = tensor_arg(a[0]), x = tensor_arg(a[1]), w = tensor_arg(a[2]), s = tensor_arg(a[3]);
        const bool nx = bool_arg(a[4]), nw = bool_arg(a[5]), nb = bool_arg(a[6]);
        return wrapped(released([&] { return norm_backward(g, x, w, s, nx, nw, nb); }));
    });
}
PyObject* py_norm(ARGS) {
    return guarded(n, 4, [&] {
        const Tensor x = tensor_arg(a[0]), w = tensor_arg(a[1]), b = tensor_arg(a[2]);
        const double eps = float_arg(a[3]);
        return wrapped(released([&] { return norm(x, w, b, eps); }));
    });
}
PyObject* py_linear_forward(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor x = tensor_arg(a[0]), w = tensor_arg(a[1]), b = tensor_arg(a[2]), r = tensor_arg(a[4]);
        const int64_t act = int_arg(a[3]), out = int_arg(a[5]);
        const bool save = bool_arg(a[6]);
        return wrapped(released([&] { return linear_forward(x, w, b, act, r, out, save); }), save);
    });
}
PyObject* py_linear_backward(ARGS) {
    return guarded(n, 8, [&] {
        const Tensor g = tensor_arg(a[0]), x = tensor_arg(a[1]), w = tensor_arg(a[2]), s = tensor_arg(a[3]);
        const int64_t act = int_arg(a[4]);
        const bool nx = bool_arg(a[5]), nw = bool_arg(a[6]), nb = bool_arg(a[7]);
        return wrapped(released([&] { return linear_backward(g, x, w, s, act, nx, nw, nb); }));
    });
}
PyObject* py_linear(ARGS) {
    return guarded(n, 6, [&] {
        const Tensor x = tensor_arg(a[0]), w = tensor_arg(a[1]), b = tensor_arg(a[2]), r = tensor_arg(a[4]);
        const int64_t act = int_arg(a[3]), out = int_arg(a[5]);
        return wrapped(released([&] { return linear(x, w, b, act, r, out); }));
    });
}
PyObject* py_gated_forward(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor x = tensor_arg(a[0]), wg = tensor_arg(a[1]), wu = tensor_arg(a[2]), bg = tensor_arg(a[3]), bu = tensor_arg(a[4]);
        const int64_t act = int_arg(a[5]);
        const bool save = bool_arg(a[6]);
        return wrapped(released([&] { return gated_forward(x, wg, wu, bg, bu, act, save); }), save);
    });
}
PyObject* py_gated_backward(ARGS) {
    return guarded(n, 9, [&] {
        const Tensor g = tensor_arg(a[0]), x = tensor_arg(a[1]), wg = tensor_arg(a[2]), wu = tensor_arg(a[3]), s = tensor_arg(a[4]);
        const int64_t act = int_arg(a[5]);
        const bool nx = bool_arg(a[6]), nw = bool_arg(a[7]), nb = bool_arg(a[8]);
        return wrapped(released([&] { return gated_backward(g, x, wg, wu, s, act, nx, nw, nb); }));
    });
}
PyObject* py_gated(ARGS) {
    return guarded(n, 6, [&] {
        const Tensor x = tensor_arg(a[0]), wg = tensor_arg(a[1]), wu = tensor_arg(a[2]), bg = tensor_arg(a[3]), bu = tensor_arg(a[4]);
        const int64_t act = int_arg(a[5]);
        return wrapped(released([&] { return gated(x, wg, wu, bg, bu, act); }));
    });
}

// p, seed (an integer or a tensor), offset
Draw draw_arg(PyObject* const* a) {
    Draw d{float_arg(a[0]), 0, 0, Tensor()};
    if (THPVariable_Check(a[1])) {
        d.state = THPVariable_Unpack(a[1]);
    } else {
        d.seed = PyLong_AsUnsignedLongLongMask(a[1]);
        if (PyErr_Occurred()) throw python_error();
    }
    d.offset = PyLong_AsUnsignedLongLongMask(a[2]);
    if (PyErr_Occurred()) throw python_error();
    return d;
}
PyObject* py_dropout_forward(ARGS) {
    return guarded(n, 5, [&] {
        const Tensor x = tensor_arg(a[0]), r = tensor_arg(a[4]);
        const Draw d = draw_arg(a + 1);
        return wrapped(released([&] { return dropout_run(x, d, r, false); }));
    });
}
PyObject* py_dropout_backward(ARGS) {
    return guarded(n, 4, [&] {
        const Tensor g = tensor_arg(a[0]);
        const Draw d = draw_arg(a + 1);
        return wrapped(released([&] { return dropout_run(g, d, Tensor(), true); }));
    });
}
PyObject* py_dropout(ARGS) {
    return guarded(n, 5, [&] {
        const Tensor x = tensor_arg(a[0]), r = tensor_arg(a[4]);
        const Draw d = draw_arg(a + 1);
        return wrapped(released([&] { return dropout(x, d, r); }));
    });
}
// weight_q, weight_k, frequencies, positions, eps
Turn turn_arg(PyObject* const* a) { return {tensor_arg(a[0]), tensor_arg(a[1]), tensor_arg(a[2]), tensor_arg(a[3]), float_arg(a[4])}; }
PyObject* py_rotary_forward(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]);
        const Turn t = turn_arg(a + 2);
        return wrapped(released([&] { return rotary_forward(q, k, t); }));
    });
}
PyObject* py_rotary_backward(ARGS) {
    return guarded(n, 11, [&] {
        const Tensor gq = tensor_arg(a[0]), gk = tensor_arg(a[1]), q = tensor_arg(a[2]), k = tensor_arg(a[3]);
        const Turn t = turn_arg(a + 4);
        const bool nx = bool_arg(a[9]), nw = bool_arg(a[10]);
        return wrapped(released([&] { return rotary_backward(gq, gk, q, k, t, nx, nw, nw); }));
    });
}
PyObject* py_rotary(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]);
        const Turn t = turn_arg(a + 2);
        return wrapped(released([&] { return rotary(q, k, t); }));
    });
}
PyObject* py_rotary_step(ARGS) {
    return guarded(n, 10, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]), v = tensor_arg(a[2]), ck = tensor_arg(a[3]), cv = tensor_arg(a[4]), l = tensor_arg(a[5]);
        const Turn t{tensor_arg(a[6]), tensor_arg(a[7]), tensor_arg(a[8]), Tensor(), float_arg(a[9])};
        return wrapped(released([&] { return rotary_step(q, k, v, ck, cv, l, t); }));
    });
}
// window, sinks, scale, lengths
Sight sight_arg(PyObject* const* a) {
    Sight s{0, int_arg(a[1]), 0, tensor_arg(a[3])};
    if (a[0] != Py_None && (s.window = int_arg(a[0])) < 1) throw Refused("window must be None or at least 1 (got " + std::to_string(s.window) + ")");
    if (a[2] != Py_None && !((s.scale = float_arg(a[2])) > 0)) throw Refused("scale must be positive (got " + std::to_string(s.scale) + ")");
    return s;
}
PyObject* py_attention_forward(ARGS) {
    return guarded(n, 8, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]), v = tensor_arg(a[2]);
        const Sight s = sight_arg(a + 3);
        const bool save = bool_arg(a[7]);
        return wrapped(released([&] { return attention_forward(q, k, v, s, save); }), save);
    });
}
PyObject* py_attention_backward(ARGS) {
    return guarded(n, 12, [&] {
        const Tensor g = tensor_arg(a[0]), q = tensor_arg(a[1]), k = tensor_arg(a[2]), v = tensor_arg(a[3]), o = tensor_arg(a[4]), l = tensor_arg(a[5]);
        const Sight s = sight_arg(a + 6);
        const bool nq = bool_arg(a[10]), nkv = bool_arg(a[11]);
        return wrapped(released([&] { return attention_backward(g, q, k, v, o, l, s, nq, nkv); }));
    });
}
PyObject* py_attention(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]), v = tensor_arg(a[2]);
        const Sight s = sight_arg(a + 3);
        return wrapped(released([&] { return attention(q, k, v, s); }));
    });
}
PyObject* py_attention_step(ARGS) {
    return guarded(n, 7, [&] {
        const Tensor q = tensor_arg(a[0]), k = tensor_arg(a[1]), v = tensor_arg(a[2]);
        const Sight s = sight_arg(a + 3);
        return wrapped(released([&] { return attention_step(q, k, v, s); }));
    });
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(norm_forward),    METHOD(norm_backward),  METHOD(norm),  METHOD(linear_forward), METHOD(linear_backward),
                          METHOD(linear),          METHOD(gated_forward),  METHOD(gated_backward), METHOD(gated),
                          METHOD(dropout_forward), METHOD(dropout_backward), METHOD(dropout), METHOD(rotary_forward), METHOD(rotary_backward),
                          METHOD(rotary),          METHOD(rotary_step),    METHOD(attention_forward), METHOD(attention_backward), METHOD(attention),
                          METHOD(attention_step), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_layers", "Native calls of paper_2607_11985_gb300.layers.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers() { return PyModule_Create(&kModule); }
