// Root-mean-square norm and rows in 8 bits on tensors.  Part of torch_binding.cpp.
#pragma once

// ---------------------------------------------------------------- rows in 8 bits

// values [..., 32 ceil(width / 32)] and scales [ceil(width / 128)][rows][4] of rows of `width`
struct InBits {
    at::Tensor values, scales;
    int64_t rows, width, ld;
};

at::ScalarType kind_type(int kind) { return kind == DGSP_E4M3 ? at::kFloat8_e4m3fn : at::kChar; }

int64_t blocks_of(int64_t width) { return (width + 31) / 32; }

constexpr int64_t kMostRowBytes = (1LL << 23) - 16;         // of the values a product reads

int64_t as_width(PyObject* o) {
    const int64_t width = as_int(o);
    if (width < 1 || width >= (1LL << 31) - 4096) refuse("width must be at least 1 and below 2^31 - 4096");
    return width;
}

InBits rows_in_8bit(const at::Tensor& values, const at::Tensor& scales, int64_t width, int kind, const char* name) {
    if (!on_gpu(values)) refuse(std::string(name) + " must hold strided tensors on the GPU");
    if (values.scalar_type() != kind_type(kind))
        refuse(std::string(name) + ".values must be " + (kind == DGSP_E4M3 ? "float8_e4m3fn" : "int8"));
    const int64_t blocks = blocks_of(width);
    if (values.dim() < 1 || values.size(-1) != 32 * blocks)
        refuse(std::string(name) + ".values must have whole blocks of 32 columns: " + std::to_string(32 * blocks) + " for a width of " + std::to_string(width));
    Rows in = rows_of(values, name);
    if (in.rows > 1 && in.ld != 0 && (in.ld % 16 != 0 || in.ld > kMostRowBytes)) in = rows_of(in.t.contiguous(), name);
    if (in.rows > 0 && reinterpret_cast<uintptr_t>(in.t.data_ptr()) % 16 != 0) in = rows_of(in.t.clone(at::MemoryFormat::Contiguous), name);
    if (!on_gpu(scales) || scales.scalar_type() != at::kByte || scales.device() != values.device() || scales.dim() != 3 ||
        scales.size(0) != (blocks + 3) / 4 || scales.size(1) != in.rows || scales.size(2) != 4)
        refuse(std::string(name) + ".scales must be uint8, ceil(width / 128) x rows x 4, on the device of the values");
    at::Tensor packed_scales = scales.contiguous();
    if (in.rows > 0 && reinterpret_cast<uintptr_t>(packed_scales.data_ptr()) % 4 != 0) packed_scales = packed_scales.clone();
    return {in.t, packed_scales, in.rows, width, in.ld};
}

InBits empty_in_8bit(at::IntArrayRef shape, int64_t rows, int kind, const at::Tensor& like) {
    const int64_t width = shape.back(), blocks = blocks_of(width);
    std::vector<int64_t> filled = shape.vec();
    filled.back() = 32 * blocks;
    return {empty_on(filled, kind_type(kind), like), empty_on({(blocks + 3) / 4, rows, 4}, at::kByte, like), rows, width, 32 * blocks};
}

InBits run_quantise(const at::Tensor& x, int kind) {
    const int type = type_of(x, "x");
    const Rows in = rows_of(x, "x");
    if (in.width < 1) refuse("the last axis of x must not be empty");
    const c10::DeviceGuard guard(x.device());
    const InBits out = empty_in_8bit(x.sizes(), in.rows, kind, x);
    check(dgsp_quantise(in.rows, in.width, type, kind, ptr(in.t), in.ld, ptr(out.values), out.ld, ptr(out.scales), stream()), "dgsp_quantise");
    return out;
}

at::ScalarType scalar_type(int type) {
    switch (type) {
        case DGSP_F32: return at::kFloat;
        case DGSP_BF16: return at::kBFloat16;
        case DGSP_F16: return at::kHalf;
        default: refuse("dtype must be float32, bfloat16 or float16");
    }
}

std::vector<int64_t> with_last(const at::Tensor& t, int64_t last) {
    std::vector<int64_t> shape = t.sizes().vec();
    shape.back() = last;
    return shape;
}

at::Tensor run_dequantise(const at::Tensor& values, const at::Tensor& scales, int64_t width, int kind, int type) {
    const at::ScalarType to = scalar_type(type);
    const c10::DeviceGuard guard(values.device());
    const InBits in = rows_in_8bit(values, scales, width, kind, "rows");
    at::Tensor y = empty_on(with_last(values, width), to, values);
    check(dgsp_dequantise(in.rows, width, type, kind, ptr(in.values), in.ld, ptr(in.scales), ptr(y), width, stream()), "dgsp_dequantise");
    return y;
}

// ---------------------------------------------------------------- the norm

Norm run_rms_norm(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& weight, float eps, const Drop& drop, const at::Tensor& offset,
                  bool want_rstd) {
    const int type = type_of(x, "x"), param_type = check_params(x, weight, {});
    const Rows in = rows_of(x, "x");
    if (in.width < 1) refuse("the last axis of x must not be empty");
    if (!(eps >= 0.0f)) refuse("eps must not be negative");
    Rows add;
    Norm out;
    const at::Tensor w = packed(weight);
    const c10::DeviceGuard guard(x.device());
    if (residual.defined()) {
        check_like(residual, x, "residual");
        if (residual.sizes() != x.sizes()) refuse("residual must have the shape of x");
        add = rows_of(residual, "residual");
        out.sum = empty_on(x.sizes(), x.scalar_type(), x);
    }
    out.y = empty_on(x.sizes(), x.scalar_type(), x);
    if (want_rstd) out.stats = empty_on(at::IntArrayRef(&in.rows, 1), at::kFloat, x);
    const dgsp_dropout_t d = drop.on(offset);
    check(dgsp_rms_norm(in.rows, in.width, type, param_type, ptr(in.t), in.ld, at_or_null(add.t), add.ld, residual.defined() ? &d : nullptr, at_or_null(w),
                        eps, ptr(out.y), in.width, at_or_null(out.sum), in.width, want_rstd ? static_cast<float*>(ptr(out.stats)) : nullptr, stream()),
          "dgsp_rms_norm");
    return out;
}

// `residual` defined: s is x.  `weight` undefined: the norm has none; `ds` undefined: none.  The gradient of x is its own tensor only
// under dropout.
NormGradient run_rms_norm_backward(const at::Tensor& s, const at::Tensor& residual, const at::Tensor& rstd, const at::Tensor& weight, const at::Tensor& dy,
                                   const at::Tensor& ds, bool dropped, const Drop& drop, const at::Tensor& offset, bool want_weight, at::ScalarType params) {
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
    check_left(rstd, at::kFloat, in.rows, s, "rstd");
    const at::Tensor w = packed(weight);
    const c10::DeviceGuard guard(s.device());
    NormGradient out;
    out.sum = empty_on(s.sizes(), s.scalar_type(), s);
    if (dropped) out.x = empty_on(s.sizes(), s.scalar_type(), s);
    const int64_t width = in.width;
    at::Tensor workspace;
    int64_t bytes = 0;
    if (want_weight) {
        out.weight = empty_on(at::IntArrayRef(&width, 1), params, s);
        bytes = dgsp_rms_norm_backward_workspace_bytes(in.rows, width);
        workspace = empty_bytes(bytes, s);
    }
    const dgsp_dropout_t d = drop.on(offset);
    check(dgsp_rms_norm_backward(in.rows, width, type, params == at::kFloat ? DGSP_F32 : type, ptr(in.t), in.ld, at_or_null(add.t), add.ld,
                                 static_cast<const float*>(ptr(rstd)), at_or_null(w), ptr(grad.t), grad.ld, at_or_null(more.t), more.ld, dropped ? &d : nullptr,
                                 ptr(out.sum), at_or_null(out.x), at_or_null(out.weight), at_or_null(workspace), bytes, stream()),
          "dgsp_rms_norm_backward");
    return out;
}

struct RmsNormBackward : public LayerNode {
    SavedDrop saved;
    SavedVariable s, added, weight, rstd;          // s: the sum, or x if the sum is made again from it and `added`
    bool residual, sum_again, has_weight;
    at::ScalarType params;
    std::string name() const override { return residual ? "AddRmsNormBackward" : "RmsNormBackward"; }
    void release_variables() override {
        for (SavedVariable* v : {&s, &added, &weight, &rstd, &saved.offset}) v->reset_data();
    }
    // edges: x, weight, and the residual
    variable_list apply(variable_list&& grads) override {
        once_only();
        variable_list out(residual ? 3 : 2);
        const at::Tensor more = residual ? grads[1] : at::Tensor();
        const Drop& drop = saved.drop;
        const at::Tensor where = saved.unpack_offset();
        const bool dropped = residual && drop.host.p > 0.0;
        if (!grads[0].defined()) {
            if (!more.defined()) return out;
            out[0] = dropped ? run_dropout(more, drop, where, {}) : more;
            out[2] = more;
            return out;
        }
        const at::Tensor sum = s.unpack(residual && !sum_again ? shared_from_this() : nullptr);
        NormGradient g = run_rms_norm_backward(sum, sum_again ? added.unpack() : at::Tensor(), rstd.unpack(), has_weight ? weight.unpack() : at::Tensor(),
                                               grads[0], more, dropped, drop, where, has_weight && task_should_compute_output(1), params);
        out[0] = dropped ? g.x : g.sum;
        out[1] = g.weight;
        if (residual) out[2] = g.sum;
        return out;
    }
};

PyObject* rms(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& weight, float eps, const Drop& drop) {
    const bool graph = wants_grad({x, residual, weight});
    Norm out;
    {
        at::NoGradGuard no_grad;
        const Unlocked unlocked;
        out = run_rms_norm(x, residual, weight, eps, drop, drop.offset, graph);
    }
    if (graph) {
        auto node = new_node<RmsNormBackward>();
        node->saved.save(drop);
        node->residual = residual.defined();
        node->sum_again = again(x, residual);
        node->has_weight = weight.defined();
        node->params = weight.defined() ? weight.scalar_type() : x.scalar_type();
        node->rstd = SavedVariable(out.stats, false);
        if (weight.defined()) node->weight = SavedVariable(weight, false);
        if (residual.defined()) {
            node->set_next_edges(torch::autograd::collect_next_edges(x, weight, residual));
            torch::autograd::set_history(out.y, node);
            torch::autograd::set_history(out.sum, node);
            if (node->sum_again) {
                node->s = SavedVariable(x, false);
                node->added = SavedVariable(residual, false);
            } else {
                node->s = SavedVariable(out.sum, true);
            }
        } else {
            node->set_next_edges(torch::autograd::collect_next_edges(x, weight));
            torch::autograd::set_history(out.y, node);
            node->s = SavedVariable(x, false);
        }
    }
    return residual.defined() ? wrap_all({out.y, out.sum}) : wrap(out.y);
}

// (x, weight, eps) -> y
PyObject* rms_norm(PyObject* const* a, Py_ssize_t n) {
    want(n, 3);
    const at::Tensor& x = as_tensor(a[0], "x");
    const at::Tensor weight = optional_tensor(a[1], "weight");
    if (!only_reverse_mode({x, weight})) Py_RETURN_NONE;
    return rms(x, {}, weight, to_float(a[2]), Drop());
}

// (x, residual, weight, eps, p, seed, offset) -> (y, s)
PyObject* add_rms_norm(PyObject* const* a, Py_ssize_t n) {
    want(n, 7);
    const at::Tensor &x = as_tensor(a[0], "x"), &residual = as_tensor(a[1], "residual");
    const at::Tensor weight = optional_tensor(a[2], "weight");
    if (!only_reverse_mode({x, residual, weight})) Py_RETURN_NONE;
    return rms(x, residual, weight, to_float(a[3]), as_drop(a + 4, x));
}

// (x, residual, weight, eps, p, seed, offset) -> (y, sum, rstd)
PyObject* rms_norm_forward(PyObject* const* a, Py_ssize_t n) {
    want(n, 7);
    const at::Tensor& x = as_tensor(a[0], "x");
    at::NoGradGuard no_grad;
    const Drop drop = as_drop(a + 4, x);
    const Norm out = run_rms_norm(x, optional_tensor(a[1], "residual"), optional_tensor(a[2], "weight"), to_float(a[3]), drop, drop.offset, true);
    return wrap_all({out.y, out.sum, out.stats});
}

// (s, residual, rstd, weight, dy, ds, dropped, p, seed, offset) -> (dsum, dx, dweight)
PyObject* rms_norm_backward(PyObject* const* a, Py_ssize_t n) {
    want(n, 10);
    const at::Tensor& s = as_tensor(a[0], "s");
    at::NoGradGuard no_grad;
    const at::Tensor weight = optional_tensor(a[3], "weight");
    const Drop drop = as_drop(a + 7, s);
    const NormGradient g = run_rms_norm_backward(s, optional_tensor(a[1], "residual"), as_tensor(a[2], "rstd"), weight, as_tensor(a[4], "dy"),
                                                 optional_tensor(a[5], "ds"), as_int(a[6]) != 0, drop, drop.offset, weight.defined(),
                                                 weight.defined() ? weight.scalar_type() : s.scalar_type());
    return wrap_all({g.sum, g.x, g.weight});
}

// What has no gradient says so.
void without_gradient(std::initializer_list<at::Tensor> inputs, const char* what) {
    if (!only_reverse_mode(inputs)) refuse(std::string(what) + " has no derivatives and takes no function transforms");
    if (wants_grad(inputs)) refuse(std::string(what) + " has no gradient: call it under torch.no_grad() or detach its inputs");
}

// (x, residual, weight, eps) -> (values, scales) or (values, scales, s)
PyObject* rms_norm_8bit(PyObject* const* a, Py_ssize_t n) {
    want(n, 4);
    const at::Tensor& x = as_tensor(a[0], "x");
    const at::Tensor residual = optional_tensor(a[1], "residual"), weight = optional_tensor(a[2], "weight");
    without_gradient({x, residual, weight}, "the norm in 8 bits");
    const float eps = to_float(a[3]);
    at::NoGradGuard no_grad;
    InBits out;
    at::Tensor sum;
    {
        const Unlocked unlocked;
        const int type = type_of(x, "x"), param_type = check_params(x, weight, {});
        const Rows in = rows_of(x, "x");
        if (in.width < 1) refuse("the last axis of x must not be empty");
        if (!(eps >= 0.0f)) refuse("eps must not be negative");
        const at::Tensor w = packed(weight);
        const c10::DeviceGuard guard(x.device());
        Rows add;
        if (residual.defined()) {
            check_like(residual, x, "residual");
            if (residual.sizes() != x.sizes()) refuse("residual must have the shape of x");
            add = rows_of(residual, "residual");
            sum = empty_on(x.sizes(), x.scalar_type(), x);
        }
        out = empty_in_8bit(x.sizes(), in.rows, DGSP_E4M3, x);
        check(dgsp_rms_norm_8bit(in.rows, in.width, type, param_type, ptr(in.t), in.ld, at_or_null(add.t), add.ld, at_or_null(w), eps, ptr(out.values), out.ld,
                                 ptr(out.scales), at_or_null(sum), in.width, stream()),
              "dgsp_rms_norm_8bit");
    }
    return sum.defined() ? wrap_all({out.values, out.scales, sum}) : wrap_all({out.values, out.scales});
}

// (x, kind) -> (values, scales)
PyObject* quantise(PyObject* const* a, Py_ssize_t n) {
    want(n, 2);
    const at::Tensor& x = as_tensor(a[0], "x");
    without_gradient({x}, "quantise");
    const int kind = (int)as_int(a[1]);
    at::NoGradGuard no_grad;
    InBits out;
    {
        const Unlocked unlocked;
        out = run_quantise(x, kind);
    }
    return wrap_all({out.values, out.scales});
}

// (values, scales, width, type) -> y
PyObject* dequantise(PyObject* const* a, Py_ssize_t n) {
    want(n, 4);
    const at::Tensor &values = as_tensor(a[0], "values"), &scales = as_tensor(a[1], "scales");
    const int64_t width = as_width(a[2]);
    const int type = (int)as_int(a[3]);
    without_gradient({values, scales}, "dequantise");
    at::NoGradGuard no_grad;
    at::Tensor y;
    {
        const Unlocked unlocked;
        y = run_dequantise(values, scales, width, values.scalar_type() == at::kChar ? DGSP_INT8 : DGSP_E4M3, type);
    }
    return wrap(y);
}
