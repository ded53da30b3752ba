// Calls from PyTorch into libdgsp_layers: argument checks, result tensors, workspaces and graph nodes.  Every step of the
// computation runs in the library.  The functions take positional arguments (the Python side, layers.py, documents them).
#include "../csrc/torch_helpers.hpp"

#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/grad_mode.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <utility>
#include <vector>

#include "../../include/dgsp_layers.h"

namespace {

using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

struct BadArgument : std::runtime_error {           // of a call, or of a graph node, where Python's lock may not be held
    using std::runtime_error::runtime_error;
};

[[noreturn]] void refuse(const std::string& what) { throw BadArgument(what); }

void check(int rc, const char* what) {
    if (rc != DGSP_OK) refuse(std::string(what) + ": " + dgsp_status_string(rc) + " (status " + std::to_string(rc) + ")");
}

int type_of(const at::Tensor& t, const char* name) {
    if (!on_gpu(t)) refuse(std::string(name) + " must be a strided tensor on the GPU");
    switch (t.scalar_type()) {
        case at::kFloat: return DGSP_F32;
        case at::kBFloat16: return DGSP_BF16;
        case at::kHalf: return DGSP_F16;
        default: refuse(std::string(name) + " must be float32, bfloat16 or float16");
    }
}

void check_like(const at::Tensor& t, const at::Tensor& x, const char* name) {
    type_of(t, name);
    if (t.scalar_type() != x.scalar_type()) refuse(std::string(name) + " must have the type of x");
    if (t.device() != x.device()) refuse(std::string(name) + " must be on the device of x");
}

// With its sign in memory: views may be marked as negative in place of being written.
at::Tensor signed_in_memory(const at::Tensor& t) { return t.is_neg() ? t.resolve_neg() : t; }

// a norm's parameter as the library reads it; undefined: there is none
at::Tensor packed(const at::Tensor& t) { return t.defined() ? signed_in_memory(t).contiguous() : t; }

// The rows of a tensor whose last axis is the width.  What lies otherwise than row after row at one distance is copied.
struct Rows {
    at::Tensor t;
    int64_t rows, width, ld;
};

Rows rows_of(const at::Tensor& any, const char* name) {
    const at::Tensor given = signed_in_memory(any);
    if (given.dim() < 1) refuse(std::string(name) + " must have at least one axis");
    const int64_t width = given.size(-1), last = given.dim() - 1;
    int64_t rows = 1;
    for (int64_t d = 0; d < last; ++d) rows *= given.size(d);
    if (given.is_contiguous()) return {given, rows, width, width};
    bool evenly = width <= 1 || given.stride(last) == 1;
    int64_t ld = width;                                // distance of the rows, from the last leading axis that has two
    bool found = false;
    int64_t next = 0;                                  // what the axis in front must be apart for the rows to go on evenly
    for (int64_t d = last - 1; d >= 0; --d) {
        if (given.size(d) == 1) continue;
        if (!found) {
            ld = given.stride(d);
            found = true;
        } else if (given.stride(d) != next) {
            evenly = false;
        }
        next = given.stride(d) * given.size(d);
    }
    if (evenly && (ld >= width || ld == 0)) return {given, rows, width, ld};
    return {given.contiguous(), rows, width, width};
}

Rows matrix_of(const at::Tensor& t, const char* name) {
    if (t.dim() != 2) refuse(std::string(name) + " must have two axes");
    return rows_of(t, name);
}

at::Tensor empty_on(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
    return at::Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt));
}

at::Tensor empty_bytes(int64_t bytes, const at::Tensor& like) {
    const int64_t n = bytes;
    return empty_on(at::IntArrayRef(&n, 1), at::kByte, like);
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

void* at_or_null(const at::Tensor& t) { return t.defined() ? ptr(t) : nullptr; }

// ---------------------------------------------------------------- dropout's arguments

struct Drop {
    dgsp_dropout_t host{0.0, 0, 0, nullptr};
    at::Tensor offset;                                 // undefined: a number of the host's
    dgsp_dropout_t on(const at::Tensor& where) const {
        dgsp_dropout_t d = host;
        d.device_offset = where.defined() ? static_cast<const uint64_t*>(where.data_ptr()) : nullptr;
        return d;
    }
};

uint64_t as_word(PyObject* o, const char* name) {
    PyObject* i = PyNumber_Index(o);
    if (!i) throw Raised{};
    const unsigned long long v = PyLong_AsUnsignedLongLong(i);
    Py_DECREF(i);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(name) + " must be at least 0 and below 2^64");
    }
    return v;
}

double as_rate(PyObject* o) {
    const double p = PyFloat_AsDouble(o);
    if (p == -1.0 && PyErr_Occurred()) throw Raised{};
    if (!(p >= 0.0 && p <= 1.0)) refuse("p must be between 0 and 1");
    return p;
}

// a[0 ... 2]: p, seed, offset
Drop as_drop(PyObject* const* a, const at::Tensor& x) {
    Drop d;
    d.host.p = as_rate(a[0]);
    d.host.seed = as_word(a[1], "seed");
    if (THPVariable_Check(a[2])) {
        d.offset = THPVariable_Unpack(a[2]);
        if (!is_array(d.offset, at::kLong) || d.offset.numel() != 1 || d.offset.device() != x.device())
            refuse("offset must be a number, or an int64 tensor of one element on the device of x");
    } else {
        d.host.offset = as_word(a[2], "offset");
    }
    return d;
}

at::Tensor optional_tensor(PyObject* o, const char* name) { return o == Py_None ? at::Tensor() : as_tensor(o, name); }

// ---------------------------------------------------------------- the library's calls on tensors

at::Tensor run_dropout(const at::Tensor& x, const Drop& drop, const at::Tensor& offset, const at::Tensor& residual) {
    const int type = type_of(x, "x");
    const Rows in = rows_of(x, "x");
    Rows add;
    if (residual.defined()) {
        check_like(residual, x, "residual");
        if (residual.sizes() != x.sizes()) refuse("residual must have the shape of x");
        add = rows_of(residual, "residual");
    }
    const c10::DeviceGuard guard(x.device());
    at::Tensor y = empty_on(x.sizes(), x.scalar_type(), x);
    const dgsp_dropout_t d = drop.on(offset);
    check(dgsp_dropout(in.rows, in.width, type, &d, ptr(in.t), in.ld, at_or_null(add.t), add.ld, ptr(y), in.width, stream()), "dgsp_dropout");
    return y;
}

struct Norm {
    at::Tensor y, sum, stats;
};

// `param_type` of the weight, the bias, or of both
int check_params(const at::Tensor& x, const at::Tensor& weight, const at::Tensor& bias) {
    const int type = type_of(x, "x");
    int param_type = type;
    for (const auto& [t, name] : {std::pair<const at::Tensor&, const char*>(weight, "weight"), {bias, "bias"}}) {
        if (!t.defined()) continue;
        param_type = type_of(t, name);
        if (param_type != type && param_type != DGSP_F32) refuse(std::string(name) + " must be float32 or have the type of x");
        if (t.dim() != 1 || x.dim() < 1 || t.size(0) != x.size(-1)) refuse(std::string(name) + " must have one axis, as long as the last of x");
        if (t.device() != x.device()) refuse(std::string(name) + " must be on the device of x");
    }
    if (weight.defined() && bias.defined() && weight.scalar_type() != bias.scalar_type()) refuse("weight and bias must have the same type");
    return param_type;
}

Norm run_norm(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& weight, const at::Tensor& bias, float eps,
              const Drop& drop, const at::Tensor& offset, bool want_stats) {
    const int type = type_of(x, "x"), param_type = check_params(x, weight, bias);
    const Rows in = rows_of(x, "x");
    if (in.width < 1) refuse("the last axis of x must not be empty");
    if (!(eps >= 0.0f)) refuse("eps must not be negative");
    Rows add;
    Norm out;
    const at::Tensor w = packed(weight), b = packed(bias);
    const c10::DeviceGuard guard(x.device());
    if (residual.defined()) {
        check_like(residual, x, "residual");
        if (residual.sizes() != x.sizes()) refuse("residual must have the shape of x");
        add = rows_of(residual, "residual");
        out.sum = empty_on(x.sizes(), x.scalar_type(), x);
    }
    out.y = empty_on(x.sizes(), x.scalar_type(), x);
    if (want_stats) {
        const int64_t n = 2 * in.rows;
        out.stats = empty_on(at::IntArrayRef(&n, 1), at::kFloat, x);
    }
    const dgsp_dropout_t d = drop.on(offset);
    check(dgsp_layer_norm(in.rows, in.width, type, param_type, ptr(in.t), in.ld, at_or_null(add.t), add.ld,
                          residual.defined() ? &d : nullptr, at_or_null(w), at_or_null(b), eps, ptr(out.y), in.width,
                          at_or_null(out.sum), in.width, want_stats ? static_cast<float*>(ptr(out.stats)) : nullptr, stream()),
          "dgsp_layer_norm");
    return out;
}

struct NormGradient {
    at::Tensor sum, x, weight, bias;
};

// What a forward pass left, as hooks of saved tensors may give it back.
void check_left(const at::Tensor& t, at::ScalarType type, int64_t count, const at::Tensor& like, const char* name) {
    if (!is_array(t, type) || t.numel() != count || t.device() != like.device()) refuse(std::string(name) + " must be what the forward pass left");
}

// Is the sum made again from x and the residual in the backward pass, where the one that was written is rounded?
bool again(const at::Tensor& x, const at::Tensor& residual) { return residual.defined() && x.scalar_type() != at::kFloat; }

// `residual` defined: s is x.  `weight` and `bias` undefined: the norm has none; `ds` undefined: none.  The gradient of x is its own tensor
// only under dropout.
NormGradient run_norm_backward(const at::Tensor& s, const at::Tensor& residual, const at::Tensor& stats, const at::Tensor& weight, const at::Tensor& dy,
                               const at::Tensor& ds, bool dropped, const Drop& drop, const at::Tensor& offset, bool want_weight,
                               bool want_bias, at::ScalarType params) {
    const int type = type_of(s, "s");
    const Rows in = rows_of(s, "s"), grad = rows_of(dy, "dy");
    check_like(dy, s, "dy");
    if (dy.sizes() != s.sizes()) refuse("dy must have the shape of s");
    Rows more, add;
    if (residual.defined()) {
        check_like(residual, s, "residual");
        if (residual.sizes() != s.sizes()) refuse("residual must have the shape of s");
        add = rows_of(residual, "residual");
    }
    if (ds.defined()) {
        check_like(ds, s, "ds");
        if (ds.sizes() != s.sizes()) refuse("ds must have the shape of s");
        more = rows_of(ds, "ds");
    }
    if (weight.defined() && weight.scalar_type() != params) refuse("weight must have the type it had");
    check_params(s, weight, {});
    check_left(stats, at::kFloat, 2 * in.rows, s, "stats");
    const at::Tensor w = packed(weight);
    const c10::DeviceGuard guard(s.device());
    NormGradient out;
    out.sum = empty_on(s.sizes(), s.scalar_type(), s);
    if (dropped) out.x = empty_on(s.sizes(), s.scalar_type(), s);
    const int64_t width = in.width;
    if (want_weight) out.weight = empty_on(at::IntArrayRef(&width, 1), params, s);
    if (want_bias) out.bias = empty_on(at::IntArrayRef(&width, 1), params, s);
    at::Tensor workspace;
    int64_t bytes = 0;
    if (want_weight || want_bias) {
        bytes = dgsp_layer_norm_backward_workspace_bytes(in.rows, width);
        workspace = empty_bytes(bytes, s);
    }
    const dgsp_dropout_t d = drop.on(offset);
    check(dgsp_layer_norm_backward(in.rows, width, type, params == at::kFloat ? DGSP_F32 : type, ptr(in.t), in.ld,
                                   at_or_null(add.t), add.ld, static_cast<const float*>(ptr(stats)), at_or_null(w), ptr(grad.t), grad.ld, at_or_null(more.t), more.ld,
                                   dropped ? &d : nullptr, ptr(out.sum), at_or_null(out.x), at_or_null(out.weight), at_or_null(out.bias),
                                   at_or_null(workspace), bytes, stream()),
          "dgsp_layer_norm_backward");
    return out;
}

struct Gated {
    Rows x, gate, up, down;
    int type, activation;
    int64_t width() const { return x.width; }
    int64_t hidden() const { return gate.rows; }
    int64_t out_width() const { return down.rows; }
};

Gated gated_arguments(const at::Tensor& x, const at::Tensor& w_gate, const at::Tensor& w_up, const at::Tensor& w_down, int activation) {
    Gated g;
    g.type = type_of(x, "x");
    g.activation = activation;
    check_like(w_gate, x, "w_gate");
    check_like(w_up, x, "w_up");
    check_like(w_down, x, "w_down");
    g.x = rows_of(x, "x");
    g.gate = matrix_of(w_gate, "w_gate");
    g.up = matrix_of(w_up, "w_up");
    g.down = matrix_of(w_down, "w_down");
    if (g.x.width < 1 || g.gate.rows < 1 || g.down.rows < 1) refuse("the block's widths must not be empty");
    if (g.gate.width != g.x.width || w_up.sizes() != w_gate.sizes()) refuse("w_gate and w_up must be hidden x width, with the last axis of x as width");
    if (g.down.width != g.gate.rows) refuse("w_down must be out_width x hidden");
    return g;
}

std::vector<int64_t> with_width(const at::Tensor& x, int64_t width) {
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = width;
    return shape;
}

std::pair<at::Tensor, at::Tensor> run_gated(const Gated& g, const at::Tensor& x, bool want_saved) {
    const c10::DeviceGuard guard(x.device());
    const int64_t rows = g.x.rows, width = g.width(), hidden = g.hidden(), out_width = g.out_width();
    at::Tensor y = empty_on(with_width(x, out_width), x.scalar_type(), x), saved, workspace;
    if (want_saved) saved = empty_bytes(dgsp_gated_ff_saved_bytes(rows, width, hidden, out_width, g.type), x);
    const int64_t bytes = dgsp_gated_ff_workspace_bytes(rows, width, hidden, out_width, g.type);
    workspace = empty_bytes(bytes, x);
    check(dgsp_gated_ff(rows, width, hidden, out_width, g.type, g.activation, ptr(g.x.t), g.x.ld, ptr(g.gate.t), g.gate.ld, ptr(g.up.t),
                        g.up.ld, ptr(g.down.t), g.down.ld, ptr(y), out_width, at_or_null(saved), ptr(workspace), bytes, stream()),
          "dgsp_gated_ff");
    return {y, saved};
}

// gradients of x, w_gate, w_up, w_down; `wanted`: which
std::vector<at::Tensor> run_gated_backward(const Gated& g, const at::Tensor& x, const at::Tensor& dy, const at::Tensor& saved,
                                           const bool (&wanted)[4]) {
    const c10::DeviceGuard guard(x.device());
    const int64_t rows = g.x.rows, width = g.width(), hidden = g.hidden(), out_width = g.out_width();
    check_like(dy, x, "dy");
    const Rows grad = rows_of(dy, "dy");
    if (grad.rows != rows || grad.width != out_width) refuse("dy must have the shape of y");
    check_left(saved, at::kByte, dgsp_gated_ff_saved_bytes(rows, width, hidden, out_width, g.type), x, "saved");
    std::vector<at::Tensor> out(4);
    if (wanted[0]) out[0] = empty_on(x.sizes(), x.scalar_type(), x);
    for (int i = 1; i < 4; ++i)
        if (wanted[i]) out[i] = empty_on(i < 3 ? at::IntArrayRef{hidden, width} : at::IntArrayRef{out_width, hidden}, x.scalar_type(), x);
    const int64_t bytes = dgsp_gated_ff_backward_workspace_bytes(rows, width, hidden, out_width, g.type);
    const at::Tensor workspace = empty_bytes(bytes, x);
    check(dgsp_gated_ff_backward(rows, width, hidden, out_width, g.type, g.activation, ptr(g.x.t), g.x.ld, ptr(g.gate.t), g.gate.ld,
                                 ptr(g.up.t), g.up.ld, ptr(g.down.t), g.down.ld, ptr(grad.t), grad.ld, ptr(saved), at_or_null(out[0]),
                                 at_or_null(out[1]), at_or_null(out[2]), at_or_null(out[3]), ptr(workspace), bytes, stream()),
          "dgsp_gated_ff_backward");
    return out;
}

// ---------------------------------------------------------------- graph nodes

// Dropout's arguments as a node keeps them.
struct SavedDrop {
    Drop drop;                          // without the tensor
    SavedVariable offset;
    bool on_gpu = false;
    void save(const Drop& d) {
        drop = d;
        drop.offset.reset();
        on_gpu = d.offset.defined();
        if (on_gpu) offset = SavedVariable(d.offset, false);
    }
    at::Tensor unpack_offset() const { return on_gpu ? offset.unpack() : at::Tensor(); }
};

bool captured() {
    const hipStream_t on = c10::hip::getCurrentHIPStream().stream();
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    return on != nullptr && hipStreamIsCapturing(on, &status) == hipSuccess && status == hipStreamCaptureStatusActive;
}

// What the nodes share: they are not differentiable themselves, as their kernels are not, and say so.  All tensors that they keep are
// SavedVariables: hooks may move them elsewhere, and changes in between are noticed.
struct LayerNode : public torch::autograd::Node {
    // Of a leaf that another graph holds, torch adds the gradients on the stream where that graph began.  From a capture it would send them to the default
    // stream, which can take part in none, and end the process; other streams join the capture.
    void once_only() const {
        TORCH_CHECK(!at::GradMode::is_enabled(), name(), ": gradients of gradients are not supported (create_graph=True)");
        if (!captured()) return;
        for (uint32_t i = 0; i < num_outputs(); ++i) {
            const auto& to = next_edge(i).function;
            if (!to || !task_should_compute_output(i)) continue;
            const auto where = to->stream();
            TORCH_CHECK(!where || where->id() != 0, name(), ": the gradient of a leaf cannot be captured while a graph made on the default stream holds the leaf");
        }
    }
};

struct DropoutBackward : public LayerNode {
    SavedDrop saved;
    bool residual;
    std::string name() const override { return "DropoutBackward"; }
    void release_variables() override { saved.offset.reset_data(); }
    variable_list apply(variable_list&& grads) override {
        once_only();
        variable_list out(residual ? 2 : 1);
        if (!grads[0].defined()) return out;
        if (task_should_compute_output(0)) out[0] = run_dropout(grads[0], saved.drop, saved.unpack_offset(), {});
        if (residual) out[1] = grads[0];
        return out;
    }
};

struct NormBackward : public LayerNode {
    SavedDrop saved;
    SavedVariable s, added, weight, stats;         // s: the sum, or x if the sum is made again from it and `added`
    bool residual, sum_again, has_weight, has_bias;
    at::ScalarType params;
    std::string name() const override { return residual ? "AddLayerNormBackward" : "LayerNormBackward"; }
    void release_variables() override {
        s.reset_data();
        added.reset_data();
        weight.reset_data();
        stats.reset_data();
        saved.offset.reset_data();
    }
    // edges: x, weight, bias, and the residual
    variable_list apply(variable_list&& grads) override {
        once_only();
        variable_list out(residual ? 4 : 3);
        const at::Tensor more = residual ? grads[1] : at::Tensor();
        const Drop& drop = saved.drop;
        const at::Tensor where = saved.unpack_offset();
        const bool dropped = residual && drop.host.p > 0.0;
        if (!grads[0].defined()) {
            if (!more.defined()) return out;
            out[0] = dropped ? run_dropout(more, drop, where, {}) : more;
            out[3] = more;
            return out;
        }
        const at::Tensor sum = s.unpack(residual && !sum_again ? shared_from_this() : nullptr);
        NormGradient g = run_norm_backward(sum, sum_again ? added.unpack() : at::Tensor(), stats.unpack(), has_weight ? weight.unpack() : at::Tensor(), grads[0], more, dropped, drop, where,
                                           has_weight && task_should_compute_output(1), has_bias && task_should_compute_output(2), params);
        out[0] = dropped ? g.x : g.sum;
        out[1] = g.weight;
        out[2] = g.bias;
        if (residual) out[3] = g.sum;
        return out;
    }
};

struct GatedBackward : public LayerNode {
    SavedVariable x, w_gate, w_up, w_down, saved;
    int activation;
    std::string name() const override { return "GatedFeedForwardBackward"; }
    void release_variables() override {
        for (SavedVariable* v : {&x, &w_gate, &w_up, &w_down, &saved}) v->reset_data();
    }
    variable_list apply(variable_list&& grads) override {
        once_only();
        if (!grads[0].defined()) return variable_list(4);
        const at::Tensor in = x.unpack();
        const Gated g = gated_arguments(in, w_gate.unpack(), w_up.unpack(), w_down.unpack(), activation);
        const bool wanted[4] = {task_should_compute_output(0), task_should_compute_output(1), task_should_compute_output(2),
                                task_should_compute_output(3)};
        return run_gated_backward(g, in, grads[0], saved.unpack(), wanted);
    }
};

template <typename N>
std::shared_ptr<N> new_node() {
    return std::shared_ptr<N>(new N(), torch::autograd::deleteNode);
}

bool wants_grad(std::initializer_list<at::Tensor> inputs) {
    if (!at::GradMode::is_enabled()) return false;
    for (const at::Tensor& t : inputs)
        if (t.defined() && t.requires_grad()) return true;
    return false;
}

bool only_reverse_mode(std::initializer_list<at::Tensor> inputs) {
    for (const at::Tensor& t : inputs)
        if (t.defined() && !only_reverse_mode(t)) return false;
    return true;
}

// ---------------------------------------------------------------- the functions

// The interpreter lock is released while the library is called: a full queue can make a launch wait.
class Unlocked {
public:
    Unlocked() : state_(PyEval_SaveThread()) {}
    ~Unlocked() { PyEval_RestoreThread(state_); }
    Unlocked(const Unlocked&) = delete;
    Unlocked& operator=(const Unlocked&) = delete;

private:
    PyThreadState* state_;
};

// As `entry`, with a refusal as the module's error.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* checked(PyObject* const* a, Py_ssize_t n) {
    try {
        return F(a, n);
    } catch (const BadArgument& e) {
        fail(e.what());
    }
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

PyObject* wrap_all(std::initializer_list<at::Tensor> ts) {
    PyObject* tuple = PyTuple_New((Py_ssize_t)ts.size());
    if (!tuple) throw Raised{};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = wrap(t);
        if (!o) {
            Py_DECREF(tuple);
            throw Raised{};
        }
        PyTuple_SET_ITEM(tuple, i++, o);
    }
    return tuple;
}

// Each of the first three: results with a graph node; None: the caller takes the way through autograd's own Function.

// (x, p, seed, offset, residual) -> y
PyObject* dropout(PyObject* const* a, Py_ssize_t n) {
    want(n, 5);
    const at::Tensor& x = as_tensor(a[0], "x");
    const at::Tensor residual = optional_tensor(a[4], "residual");
    if (!only_reverse_mode({x, residual})) Py_RETURN_NONE;
    const Drop drop = as_drop(a + 1, x);
    at::Tensor y;
    {
        at::NoGradGuard no_grad;
        const Unlocked unlocked;
        y = run_dropout(x, drop, drop.offset, residual);
    }
    if (wants_grad({x, residual})) {
        auto node = new_node<DropoutBackward>();
        node->residual = residual.defined();
        node->saved.save(drop);
        node->set_next_edges(residual.defined() ? torch::autograd::collect_next_edges(x, residual) : torch::autograd::collect_next_edges(x));
        torch::autograd::set_history(y, node);
    }
    return wrap(y);
}

PyObject* norm(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& weight, const at::Tensor& bias, float eps, const Drop& drop) {
    const bool graph = wants_grad({x, residual, weight, bias});
    Norm out;
    {
        at::NoGradGuard no_grad;
        const Unlocked unlocked;
        out = run_norm(x, residual, weight, bias, eps, drop, drop.offset, graph);
    }
    if (graph) {
        auto node = new_node<NormBackward>();
        node->saved.save(drop);
        node->residual = residual.defined();
        node->sum_again = again(x, residual);
        node->has_weight = weight.defined();
        node->has_bias = bias.defined();
        node->params = weight.defined() ? weight.scalar_type() : bias.defined() ? bias.scalar_type() : x.scalar_type();
        node->stats = SavedVariable(out.stats, false);
        if (weight.defined()) node->weight = SavedVariable(weight, false);
        if (residual.defined()) {
            node->set_next_edges(torch::autograd::collect_next_edges(x, weight, bias, residual));
            torch::autograd::set_history(out.y, node);
            torch::autograd::set_history(out.sum, node);
            if (node->sum_again) {
                node->s = SavedVariable(x, false);
                node->added = SavedVariable(residual, false);
            } else {
                node->s = SavedVariable(out.sum, true);
            }
        } else {
            node->set_next_edges(torch::autograd::collect_next_edges(x, weight, bias));
            torch::autograd::set_history(out.y, node);
            node->s = SavedVariable(x, false);
        }
    }
    return residual.defined() ? wrap_all({out.y, out.sum}) : wrap(out.y);
}

// (x, weight, bias, eps) -> y
PyObject* layer_norm(PyObject* const* a, Py_ssize_t n) {
    want(n, 4);
    const at::Tensor& x = as_tensor(a[0], "x");
    const at::Tensor weight = optional_tensor(a[1], "weight"), bias = optional_tensor(a[2], "bias");
    if (!only_reverse_mode({x, weight, bias})) Py_RETURN_NONE;
    return norm(x, {}, weight, bias, to_float(a[3]), Drop());
}

// (x, residual, weight, bias, eps, p, seed, offset) -> (y, s)
PyObject* add_layer_norm(PyObject* const* a, Py_ssize_t n) {
    want(n, 8);
    const at::Tensor &x = as_tensor(a[0], "x"), &residual = as_tensor(a[1], "residual");
    const at::Tensor weight = optional_tensor(a[2], "weight"), bias = optional_tensor(a[3], "bias");
    if (!only_reverse_mode({x, residual, weight, bias})) Py_RETURN_NONE;
    return norm(x, residual, weight, bias, to_float(a[4]), as_drop(a + 5, x));
}

// (x, w_gate, w_up, w_down, activation) -> y
PyObject* gated_ff(PyObject* const* a, Py_ssize_t n) {
    want(n, 5);
    const at::Tensor &x = as_tensor(a[0], "x"), &w_gate = as_tensor(a[1], "w_gate"), &w_up = as_tensor(a[2], "w_up"),
                     &w_down = as_tensor(a[3], "w_down");
    if (!only_reverse_mode({x, w_gate, w_up, w_down})) Py_RETURN_NONE;
    const bool graph = wants_grad({x, w_gate, w_up, w_down});
    const int activation = (int)as_int(a[4]);
    std::pair<at::Tensor, at::Tensor> out;
    {
        at::NoGradGuard no_grad;
        const Unlocked unlocked;
        out = run_gated(gated_arguments(x, w_gate, w_up, w_down, activation), x, graph);
    }
    if (graph) {
        auto node = new_node<GatedBackward>();
        node->activation = activation;
        node->saved = SavedVariable(out.second, false);
        node->x = SavedVariable(x, false);
        node->w_gate = SavedVariable(w_gate, false);
        node->w_up = SavedVariable(w_up, false);
        node->w_down = SavedVariable(w_down, false);
        node->set_next_edges(torch::autograd::collect_next_edges(x, w_gate, w_up, w_down));
        torch::autograd::set_history(out.first, node);
    }
    return wrap(out.first);
}

// The steps without a graph, for autograd's own Function.

// (x, residual, weight, bias, eps, p, seed, offset) -> (y, sum, stats)
PyObject* layer_norm_forward(PyObject* const* a, Py_ssize_t n) {
    want(n, 8);
    const at::Tensor& x = as_tensor(a[0], "x");
    at::NoGradGuard no_grad;
    const Drop drop = as_drop(a + 5, x);
    const Norm out = run_norm(x, optional_tensor(a[1], "residual"), optional_tensor(a[2], "weight"), optional_tensor(a[3], "bias"),
                              to_float(a[4]), drop, drop.offset, true);
    return wrap_all({out.y, out.sum, out.stats});
}

// (s, residual, stats, weight, bias, dy, ds, dropped, p, seed, offset) -> (dsum, dx, dweight, dbias)
PyObject* layer_norm_backward(PyObject* const* a, Py_ssize_t n) {
    want(n, 11);
    const at::Tensor& s = as_tensor(a[0], "s");
    at::NoGradGuard no_grad;
    const at::Tensor weight = optional_tensor(a[3], "weight"), bias = optional_tensor(a[4], "bias");
    const Drop drop = as_drop(a + 8, s);
    const at::ScalarType params = weight.defined() ? weight.scalar_type() : bias.defined() ? bias.scalar_type() : s.scalar_type();
    const NormGradient g = run_norm_backward(s, optional_tensor(a[1], "residual"), as_tensor(a[2], "stats"), weight, as_tensor(a[5], "dy"),
                                             optional_tensor(a[6], "ds"), as_int(a[7]) != 0, drop, drop.offset, weight.defined(), bias.defined(), params);
    return wrap_all({g.sum, g.x, g.weight, g.bias});
}

// (x, p, seed, offset, residual) -> y
PyObject* dropout_forward(PyObject* const* a, Py_ssize_t n) {
    want(n, 5);
    const at::Tensor& x = as_tensor(a[0], "x");
    at::NoGradGuard no_grad;
    const Drop drop = as_drop(a + 1, x);
    return wrap(run_dropout(x, drop, drop.offset, optional_tensor(a[4], "residual")));
}

// (x, w_gate, w_up, w_down, activation) -> (y, saved)
PyObject* gated_ff_forward(PyObject* const* a, Py_ssize_t n) {
    want(n, 5);
    at::NoGradGuard no_grad;
    const at::Tensor& x = as_tensor(a[0], "x");
    const auto out = run_gated(gated_arguments(x, as_tensor(a[1], "w_gate"), as_tensor(a[2], "w_up"), as_tensor(a[3], "w_down"),
                                               (int)as_int(a[4])), x, true);
    return wrap_all({out.first, out.second});
}

// (x, w_gate, w_up, w_down, activation, dy, saved) -> gradients of x, w_gate, w_up, w_down
PyObject* gated_ff_backward(PyObject* const* a, Py_ssize_t n) {
    want(n, 7);
    at::NoGradGuard no_grad;
    const at::Tensor& x = as_tensor(a[0], "x");
    const Gated g = gated_arguments(x, as_tensor(a[1], "w_gate"), as_tensor(a[2], "w_up"), as_tensor(a[3], "w_down"), (int)as_int(a[4]));
    const auto out = run_gated_backward(g, x, as_tensor(a[5], "dy"), as_tensor(a[6], "saved"), {true, true, true, true});
    return wrap_all({out[0], out[1], out[2], out[3]});
}

#include "torch_rms_norm.hpp"

#include "torch_linear.hpp"

#define LAYERS_ENTRY(name) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&entry<checked<name>>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    {"set_error_type", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&entry<set_error_type>)), METH_FASTCALL, nullptr},
    LAYERS_ENTRY(dropout), LAYERS_ENTRY(layer_norm), LAYERS_ENTRY(add_layer_norm), LAYERS_ENTRY(gated_ff), LAYERS_ENTRY(layer_norm_forward),
    LAYERS_ENTRY(layer_norm_backward), LAYERS_ENTRY(dropout_forward), LAYERS_ENTRY(gated_ff_forward), LAYERS_ENTRY(gated_ff_backward),
    LAYERS_ENTRY(rms_norm), LAYERS_ENTRY(add_rms_norm), LAYERS_ENTRY(rms_norm_forward), LAYERS_ENTRY(rms_norm_backward), LAYERS_ENTRY(rms_norm_8bit),
    LAYERS_ENTRY(quantise), LAYERS_ENTRY(dequantise), LAYERS_ENTRY(linear), LAYERS_ENTRY(linear_forward), LAYERS_ENTRY(linear_backward),
    LAYERS_ENTRY(linear_8bit),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_dgsp_layers_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dgsp_layers_torch(void) { return PyModule_Create(&g_module); }
