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
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

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

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(norm_forward),    METHOD(norm_backward),  METHOD(norm),  METHOD(linear_forward), METHOD(linear_backward),
                          METHOD(linear),          METHOD(gated_forward),  METHOD(gated_backward), METHOD(gated), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_layers", "Native calls of paper_2607_11985_gb300.layers.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers() { return PyModule_Create(&kModule); }
