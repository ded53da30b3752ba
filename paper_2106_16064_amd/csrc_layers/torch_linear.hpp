// The matrix product with its epilogue on tensors.  Part of torch_binding.cpp.
#pragma once

struct LinearCall {
    Rows x, weight, residual;
    at::Tensor bias;
    int type, bias_type, activation, keep;
    int64_t rows() const { return x.rows; }
    int64_t width() const { return x.width; }
    int64_t out_width() const { return weight.rows; }
};

// `bias_type` of a product's results
int check_bias(const at::Tensor& bias, int type, int64_t out_width, const at::Tensor& x) {
    if (!bias.defined()) return type;
    const int bias_type = type_of(bias, "bias");
    if (bias_type != type && bias_type != DGSP_F32) refuse("bias must be float32 or have the type of the result");
    if (bias.dim() != 1 || bias.size(0) != out_width) refuse("bias must have one axis, as long as the first of the weight");
    if (bias.device() != x.device()) refuse("bias must be on the device of x");
    return bias_type;
}

Rows check_residual(const at::Tensor& residual, at::ScalarType type, const at::Tensor& x, int64_t out_width) {
    if (!residual.defined()) return {};
    type_of(residual, "residual");
    if (residual.scalar_type() != type) refuse("residual must have the type of the result");
    if (residual.device() != x.device()) refuse("residual must be on the device of x");
    if (residual.sizes() != at::IntArrayRef(with_last(x, out_width))) refuse("residual must have the shape of the result");
    return rows_of(residual, "residual");
}

LinearCall linear_arguments(const at::Tensor& x, const at::Tensor& weight, const at::Tensor& bias, int activation, const at::Tensor& residual, int keep) {
    LinearCall c;
    c.type = type_of(x, "x");
    c.activation = activation;
    c.keep = keep;
    check_like(weight, x, "weight");
    c.x = rows_of(x, "x");
    c.weight = matrix_of(weight, "weight");
    if (c.x.width < 1 || c.weight.rows < 1) refuse("the product's widths must not be empty");
    if (c.weight.width != c.x.width) refuse("weight must be out_width x width, with the last axis of x as width");
    c.bias_type = check_bias(bias, c.type, c.weight.rows, x);
    c.bias = packed(bias);
    c.residual = check_residual(residual, x.scalar_type(), x, c.weight.rows);
    return c;
}

struct LinearResult {
    at::Tensor y, saved;        // what is left of z
    InBits x;                   // x in 8 bits, if it is wanted
};

LinearResult run_linear(const LinearCall& c, const at::Tensor& x, bool x_in_8bit) {
    const c10::DeviceGuard guard(x.device());
    const int64_t rows = c.rows(), width = c.width(), out_width = c.out_width();
    at::Tensor y = empty_on(with_last(x, out_width), x.scalar_type(), x), saved;
    const int64_t kept = dgsp_linear_saved_bytes(rows, out_width, c.type, c.bias_type, c.activation, c.keep);
    if (c.keep != DGSP_KEEP_NOTHING) saved = empty_bytes(kept, x);
    const int64_t bytes = dgsp_linear_workspace_bytes(rows, width, out_width, c.type);
    const at::Tensor workspace = bytes ? empty_bytes(bytes, x) : at::Tensor();
    const InBits in_8bit = x_in_8bit ? empty_in_8bit(x.sizes(), rows, DGSP_INT8, x) : InBits{};
    check(dgsp_linear(rows, width, out_width, c.type, c.bias_type, c.activation, c.keep, ptr(c.x.t), c.x.ld, ptr(c.weight.t), c.weight.ld, at_or_null(c.bias),
                      at_or_null(c.residual.t), c.residual.ld, ptr(y), out_width, at_or_null(saved), at_or_null(in_8bit.values), in_8bit.ld,
                      at_or_null(in_8bit.scales), at_or_null(workspace), bytes, stream()),
          "dgsp_linear");
    return {y, saved, in_8bit};
}

struct LinearGradient {
    at::Tensor x, weight, bias;
};

// `x`: the matrix, or its values in 8 bits with `scales`, undefined if the weight's gradient is not wanted; `weight` undefined: that of x is
// not; `saved`: what the forward pass left.
LinearGradient run_linear_backward(const at::Tensor& x, const at::Tensor& scales, const at::Tensor& weight, const at::Tensor& saved, const at::Tensor& dy,
                                   at::ScalarType bias_type, int activation, int keep, int64_t width, bool want_x, bool want_weight, bool want_bias) {
    if (!want_x && !want_weight && !want_bias) return {};
    const int type = type_of(dy, "dy");
    const Rows grad = rows_of(dy, "dy");
    const int64_t rows = grad.rows, out_width = grad.width;
    const c10::DeviceGuard guard(dy.device());
    Rows in, w;
    at::Tensor in_scales;
    if (want_weight && keep == DGSP_KEEP_8BIT) {
        const InBits kept = rows_in_8bit(x, scales, width, DGSP_INT8, "what the forward pass left of x");
        in = {kept.values, kept.rows, width, kept.ld};
        in_scales = kept.scales;
    } else if (want_weight) {
        check_like(x, dy, "x");
        in = rows_of(x, "x");
    }
    if (want_weight && (in.t.device() != dy.device() || in.rows != rows || in.width != width)) refuse("x must be what the forward pass left");
    if (want_x) {
        check_like(weight, dy, "weight");
        w = matrix_of(weight, "weight");
        if (w.rows != out_width || w.width != width) refuse("weight must have the shape it had");
    }
    const int to = bias_type == at::kFloat ? DGSP_F32 : type;
    const int64_t kept = dgsp_linear_saved_bytes(rows, out_width, type, to, activation, keep);
    if (kept) check_left(saved, at::kByte, kept, dy, "saved");
    LinearGradient out;
    if (want_x) out.x = empty_on(with_last(dy, width), dy.scalar_type(), dy);
    if (want_weight) out.weight = empty_on({out_width, width}, dy.scalar_type(), dy);
    if (want_bias) out.bias = empty_on(at::IntArrayRef(&out_width, 1), bias_type, dy);
    const int64_t bytes = dgsp_linear_backward_workspace_bytes(rows, width, out_width, type, activation, keep);
    const at::Tensor workspace = bytes ? empty_bytes(bytes, dy) : at::Tensor();
    check(dgsp_linear_backward(rows, width, out_width, type, to, activation, keep, at_or_null(in.t), in.ld,
                               at_or_null(in_scales), at_or_null(w.t), w.ld, at_or_null(saved), ptr(grad.t), grad.ld, at_or_null(out.x), at_or_null(out.weight),
                               at_or_null(out.bias), at_or_null(workspace), bytes, stream()),
          "dgsp_linear_backward");
    return out;
}

struct LinearBackward : public LayerNode {
    SavedVariable x, scales, weight, saved;
    int activation, keep;
    int64_t width;
    bool has_residual, has_bias, keeps_x, keeps_weight, keeps_saved;
    at::ScalarType bias_type;
    std::string name() const override { return "LinearBackward"; }
    void release_variables() override {
        for (SavedVariable* v : {&x, &scales, &weight, &saved}) v->reset_data();
    }
    // edges: x, weight, bias, residual
    variable_list apply(variable_list&& grads) override {
        once_only();
        variable_list out(4);
        const at::Tensor& dy = grads[0];
        if (!dy.defined()) return out;
        if (has_residual) out[3] = dy;
        const LinearGradient g = run_linear_backward(keeps_x ? x.unpack() : at::Tensor(), keeps_x && keep == DGSP_KEEP_8BIT ? scales.unpack() : at::Tensor(),
                                                     keeps_weight ? weight.unpack() : at::Tensor(), keeps_saved ? saved.unpack() : at::Tensor(), dy, bias_type,
                                                     activation, keep, width, keeps_weight && task_should_compute_output(0),
                                                     keeps_x && task_should_compute_output(1), has_bias && task_should_compute_output(2));
        out[0] = g.x;
        out[1] = g.weight;
        out[2] = g.bias;
        return out;
    }
};

bool asks_gradient(const at::Tensor& t) { return t.defined() && t.requires_grad(); }

// (x, weight, bias, activation, residual, keep_8bit) -> y
PyObject* linear(PyObject* const* a, Py_ssize_t n) {
    want(n, 6);
    const at::Tensor &x = as_tensor(a[0], "x"), &weight = as_tensor(a[1], "weight");
    const at::Tensor bias = optional_tensor(a[2], "bias"), residual = optional_tensor(a[4], "residual");
    if (!only_reverse_mode({x, weight, bias, residual})) Py_RETURN_NONE;
    const int activation = (int)as_int(a[3]);
    const bool in_8bit = as_int(a[5]) != 0, graph = wants_grad({x, weight, bias, residual});
    const bool of_x = graph && asks_gradient(x), of_weight = graph && asks_gradient(weight), of_bias = graph && asks_gradient(bias);
    const int keep = !(of_x || of_weight || of_bias) ? DGSP_KEEP_NOTHING : in_8bit ? DGSP_KEEP_8BIT : DGSP_KEEP_WHOLE;
    LinearResult out;
    {
        at::NoGradGuard no_grad;
        const Unlocked unlocked;
        out = run_linear(linear_arguments(x, weight, bias, activation, residual, keep), x, of_weight && in_8bit);
    }
    if (graph) {
        auto node = new_node<LinearBackward>();
        node->activation = activation;
        node->keep = in_8bit ? DGSP_KEEP_8BIT : DGSP_KEEP_WHOLE;
        node->width = x.size(-1);
        node->has_residual = residual.defined();
        node->has_bias = bias.defined();
        node->bias_type = bias.defined() ? bias.scalar_type() : x.scalar_type();
        node->keeps_x = of_weight;
        node->keeps_weight = of_x;
        node->keeps_saved = out.saved.defined();
        if (of_weight && in_8bit) {
            node->x = SavedVariable(out.x.values, false);
            node->scales = SavedVariable(out.x.scales, false);
        } else if (of_weight) {
            node->x = SavedVariable(x, false);
        }
        if (of_x) node->weight = SavedVariable(weight, false);
        if (node->keeps_saved) node->saved = SavedVariable(out.saved, false);
        node->set_next_edges(torch::autograd::collect_next_edges(x, weight, bias, residual));
        torch::autograd::set_history(out.y, node);
    }
    return wrap(out.y);
}

// (x, weight, bias, activation, residual, keep_8bit) -> (y, saved, values and scales of x or None)
PyObject* linear_forward(PyObject* const* a, Py_ssize_t n) {
    want(n, 6);
    const at::Tensor& x = as_tensor(a[0], "x");
    at::NoGradGuard no_grad;
    const bool in_8bit = as_int(a[5]) != 0;
    const LinearResult out = run_linear(linear_arguments(x, as_tensor(a[1], "weight"), optional_tensor(a[2], "bias"), (int)as_int(a[3]), optional_tensor(a[4], "residual"),
                                                 in_8bit ? DGSP_KEEP_8BIT : DGSP_KEEP_WHOLE), x, in_8bit);
    return wrap_all({out.y, out.saved, out.x.values, out.x.scales});
}

// (x or values, scales, weight, bias, saved, dy, activation) -> (dx, dweight, dbias)
PyObject* linear_backward(PyObject* const* a, Py_ssize_t n) {
    want(n, 7);
    at::NoGradGuard no_grad;
    const at::Tensor scales = optional_tensor(a[1], "scales"), bias = optional_tensor(a[3], "bias");
    const at::Tensor &weight = as_tensor(a[2], "weight"), &dy = as_tensor(a[5], "dy");
    if (weight.dim() != 2) refuse("weight must have two axes");
    const LinearGradient g = run_linear_backward(as_tensor(a[0], "x"), scales, weight, as_tensor(a[4], "saved"), dy,
                                                 bias.defined() ? bias.scalar_type() : dy.scalar_type(), (int)as_int(a[6]),
                                                 scales.defined() ? DGSP_KEEP_8BIT : DGSP_KEEP_WHOLE, weight.size(1), true, true, bias.defined());
    return wrap_all({g.x, g.weight, g.bias});
}

// (values, scales and width of x, values, scales and width of the weight, bias, activation, residual, type) -> y
PyObject* linear_8bit(PyObject* const* a, Py_ssize_t n) {
    want(n, 10);
    const at::Tensor &x = as_tensor(a[0], "x.values"), &x_scales = as_tensor(a[1], "x.scales"), &weight = as_tensor(a[3], "weight.values"),
                     &weight_scales = as_tensor(a[4], "weight.scales");
    const int64_t width = as_width(a[2]), weight_width = as_width(a[5]);
    const at::Tensor bias = optional_tensor(a[6], "bias"), residual = optional_tensor(a[8], "residual");
    const int activation = (int)as_int(a[7]), type = (int)as_int(a[9]);
    without_gradient({x, x_scales, weight, weight_scales, bias, residual}, "the product in 8 bits");
    at::NoGradGuard no_grad;
    at::Tensor y;
    {
        const Unlocked unlocked;
        const at::ScalarType to = scalar_type(type);
        const c10::DeviceGuard guard(x.device());
        const InBits in = rows_in_8bit(x, x_scales, width, DGSP_E4M3, "x"), w = rows_in_8bit(weight, weight_scales, weight_width, DGSP_E4M3, "weight");
        if (weight.dim() != 2) refuse("weight must have two axes");
        if (weight_width != width) refuse("weight must have the width of x");
        if (w.values.device() != in.values.device()) refuse("weight must be on the device of x");
        if (w.rows < 1) refuse("the product's widths must not be empty");
        const int bias_type = check_bias(bias, type, w.rows, x);
        const at::Tensor b = packed(bias);
        const Rows add = check_residual(residual, to, x, w.rows);
        y = empty_on(with_last(x, w.rows), to, x);
        const int64_t bytes = dgsp_linear_8bit_workspace_bytes(in.rows, width, w.rows);
        const at::Tensor workspace = bytes ? empty_bytes(bytes, x) : at::Tensor();
        check(dgsp_linear_8bit(in.rows, width, w.rows, type, bias_type, activation, ptr(in.values), in.ld, ptr(in.scales), ptr(w.values), w.ld, ptr(w.scales),
                               at_or_null(b), at_or_null(add.t), add.ld, ptr(y), w.rows, at_or_null(workspace), bytes, stream()),
              "dgsp_linear_8bit");
    }
    return wrap(y);
}
