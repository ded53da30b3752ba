"""Calls at the edges of what the layers take: batches without rows, one row at any distance, values at the ends of a type's range, saved
tensors that a program moves or changes."""
import pytest
import torch

from paper_2106_16064_amd import layers

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def show(*case):
    print("[case]", *case, flush=True)


# ---------------------------------------------------------------- no rows

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,hidden,out", [(1024, 2048, 1024), (2048, 40, 24), (24, 2048, 40), (40, 24, 2048)])
def test_a_deep_block_of_no_rows(width, hidden, out, dtype):
    """Results without rows, gradients of the weights that are sums of nothing."""
    show("no rows", width, hidden, out, dtype)
    x = torch.empty((2, 0, width), device="cuda", dtype=dtype, requires_grad=True)
    w = [torch.randn(shape, device="cuda").to(dtype).requires_grad_(True) for shape in ((hidden, width), (hidden, width), (out, hidden))]
    with torch.no_grad():
        assert layers.gated_ff(x, *w).shape == (2, 0, out)
    y = layers.gated_ff(x, *w)
    assert y.shape == (2, 0, out) and y.dtype == dtype
    dx, *dw = torch.autograd.grad(y, [x, *w], torch.empty_like(y))
    assert dx.shape == x.shape
    assert all(g.shape == t.shape and g.dtype == dtype and not g.any() for g, t in zip(dw, w))


# ---------------------------------------------------------------- the C interface: one row

CODES = {torch.float32: layers.F32, torch.bfloat16: layers.BF16, torch.float16: layers.F16}


def c_block(x, w, dy, ldx, lddy):
    """Result and gradients through the C entry points, with the distances of rows given."""
    L, code = layers.lib(), CODES[x.dtype]
    (rows, width), (hidden, _), (out, _) = x.shape, w[0].shape, w[2].shape
    extents = (rows, width, hidden, out, code)
    stream = torch.cuda.current_stream().cuda_stream

    def space(size):
        return torch.empty(max(size(*extents), 16), dtype=torch.uint8, device="cuda")

    saved, work, back = space(L.dgsp_gated_ff_saved_bytes), space(L.dgsp_gated_ff_workspace_bytes), space(L.dgsp_gated_ff_backward_workspace_bytes)
    y = torch.empty((rows, out), dtype=x.dtype, device="cuda")
    grads = [torch.empty_like(t) for t in (x, *w)]
    matrices = [x.data_ptr(), ldx, w[0].data_ptr(), width, w[1].data_ptr(), width, w[2].data_ptr(), hidden]
    assert L.dgsp_gated_ff(*extents, layers.SILU, *matrices, y.data_ptr(), out, saved.data_ptr(), work.data_ptr(), work.numel(), stream) == 0
    assert L.dgsp_gated_ff_backward(*extents, layers.SILU, *matrices, dy.data_ptr(), lddy, saved.data_ptr(), *(g.data_ptr() for g in grads),
                                    back.data_ptr(), back.numel(), stream) == 0
    return [y, *grads]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,hidden", [(32, 64), (32, 128), (32, 256), (64, 64), (64, 128), (64, 256), (128, 64), (128, 128), (40, 64), (256, 512)])
def test_one_row_of_a_block_has_no_distance_to_the_next(width, hidden, dtype):
    """Whatever the caller gives for it, the results are the same."""
    show("one row", width, hidden, dtype)
    torch.manual_seed(0)
    x, dy = (torch.randn((1, width), device="cuda").to(dtype) for _ in range(2))
    w = [(torch.randn(shape, device="cuda") * shape[1] ** -0.5).to(dtype) for shape in ((hidden, width), (hidden, width), (width, hidden))]
    want = c_block(x, w, dy, width, width)
    for ldx, lddy in ((8, 8), (8, width), (width, 8), (16, 24), (0, 0), (1, 1), (-8, -8), (1 << 40, 1 << 40)):
        got = c_block(x, w, dy, ldx, lddy)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (ldx, lddy)


# ---------------------------------------------------------------- gates at the ends of the range

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("hidden", [1, 300])
@pytest.mark.parametrize("activation", ["silu", "gelu", "relu"])
def test_gates_far_from_zero(activation, hidden, dtype):
    """One hidden value with g = x0 + x1, u = x2 = 1 and y = act(g), so that dx0 is act'(g).  From 88 on act(g) is g or 0 and its derivative
    1 or 0, to less than 89 2^-126 (silu of -88); h and y are rounded once each, and so are dg and dx.  The sum of the two largest is beyond
    the range of the sums, and its value too."""
    show("far gates", activation, hidden, dtype)
    ends = [88.0, 89.0, 104.0, 300.0, 1e3, 6e4] + ([1e10, 1e20, 1e30, 2.2e38, 2.5e38, 3e38] if dtype != torch.float16 else [])
    g = torch.tensor([s * v for v in ends for s in (1.0, -1.0)]).to(dtype)
    x = torch.zeros((len(g) + 1, 3), dtype=dtype)
    x[:-1, 0], x[:, 2] = g, 1.0
    x[-1, :2] = torch.finfo(dtype).max if dtype != torch.float16 else 3e4
    w_gate, w_up, w_down = torch.zeros((hidden, 3)), torch.zeros((hidden, 3)), torch.zeros((1, hidden))
    w_gate[0, :2], w_up[0, 2], w_down[0, 0] = 1.0, 1.0, 1.0
    leaf, *w = (t.cuda().to(dtype).requires_grad_(True) for t in (x, w_gate, w_up, w_down))
    y = layers.gated_ff(leaf, *w, activation=activation)
    slope, = torch.autograd.grad(y[:-1], leaf, torch.ones_like(y[:-1]))
    y, slope, want = y.detach()[:, 0].double().cpu(), slope[:-1, 0].double().cpu(), g.double().clamp(min=0.0)
    tiny = 89 * 2.0 ** -126 if dtype != torch.float16 else 2.0 ** -25
    assert ((y[:-1] - want).abs() <= 2 * UNIT[dtype] * want + tiny).all(), (g, y)
    assert ((slope - (want > 0).double()).abs() <= 4 * UNIT[dtype]).all(), (g, slope)
    if dtype == torch.float32:
        assert not torch.isfinite(y[-1])                     # an infinity among products of parts: it or NaN, which is not said
    else:
        assert y[-1] == (float("inf") if dtype == torch.bfloat16 else 6e4)


# ---------------------------------------------------------------- what the backward pass finds changed

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("which", ["add_layer_norm", "dropout"])
def test_an_offset_changed_before_the_backward_pass_is_noticed(which, dtype):
    """Another offset is another mask; on the way of the graph nodes and on that of autograd's own Functions.  Unchanged, both give what a
    number gives."""
    show("changed offset", which, dtype)
    torch.manual_seed(0)
    x, r, g = (torch.randn((20, 24), device="cuda").to(dtype) for _ in range(3))
    functions = layers._functions()
    calls = {"add_layer_norm": (lambda a, b, o: layers.add_layer_norm(a, b, p=0.5, seed=1, offset=o)[0],
                                lambda a, b, o: functions.norm.apply(a, b, None, None, 1e-5, 0.5, 1, o)[0]),
             "dropout": (lambda a, b, o: layers.dropout(a, 0.5, 1, o, residual=b), lambda a, b, o: functions.dropout.apply(a, 0.5, 1, o, b))}
    for call in calls[which]:
        leaves = [t.clone().requires_grad_(True) for t in (x, r)]
        want = torch.autograd.grad(call(*leaves, 3), leaves, g)
        offset = torch.full((1,), 3, dtype=torch.int64, device="cuda")
        got = torch.autograd.grad(call(*leaves, offset), leaves, g)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        y = call(*leaves, offset)
        offset.add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            torch.autograd.grad(y, leaves, g)


# ---------------------------------------------------------------- what the graph keeps

def layer_calls(dtype):
    """Name, call and its inputs: blocks on the general and on the narrow way."""
    torch.manual_seed(0)

    def tensors(*shapes):
        return [torch.randn(shape, device="cuda").to(dtype) for shape in shapes]

    return {
        "layer_norm": (layers.layer_norm, tensors((30, 40), (40,), (40,))),
        "add_layer_norm": (lambda *t: layers.add_layer_norm(*t, p=0.25, seed=1), tensors((30, 40), (30, 40), (40,), (40,))),
        "dropout": (lambda *t: layers.dropout(t[0], 0.25, 1, residual=t[1]), tensors((30, 40), (30, 40))),
        "narrow block": (layers.gated_ff, tensors((30, 40), (24, 40), (24, 40), (16, 24))),
        "block": (layers.gated_ff, tensors((30, 40), (300, 40), (300, 40), (16, 300))),
    }


def results(call, inputs):
    leaves = [t.clone().requires_grad_(True) for t in inputs]
    out = call(*leaves)
    out = out if isinstance(out, tuple) else (out,)
    return out, leaves


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("name", ["layer_norm", "add_layer_norm", "dropout", "narrow block", "block"])
def test_all_that_a_node_keeps_goes_through_the_hooks_of_saved_tensors(name, dtype):
    """A program may move it to the host until the backward pass or make it again then: once the results are gone, nothing of the call is
    left on the GPU, and the gradients are the same."""
    show("saved tensors", name, dtype)
    call, inputs = layer_calls(dtype)[name]
    out, leaves = results(call, inputs)
    grads = [torch.randn_like(t) for t in out]
    want = torch.autograd.grad(out, leaves, grads)

    with torch.autograd.graph.save_on_cpu():
        out, leaves = results(call, inputs)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, grads), want))

    from torch.utils.checkpoint import checkpoint
    leaves = [t.clone().requires_grad_(True) for t in inputs]
    out = checkpoint(call, *leaves, use_reentrant=False)
    out = out if isinstance(out, tuple) else (out,)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, grads), want))
    del out, leaves, want

    leaves = [t.clone().requires_grad_(True) for t in inputs]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    with torch.autograd.graph.save_on_cpu():
        out = call(*leaves)
    nodes = {t.grad_fn for t in (out if isinstance(out, tuple) else (out,))}
    assert len(nodes) == 1
    del out
    assert torch.cuda.memory_allocated() == before
    del nodes


@pytest.mark.parametrize("name", ["layer_norm", "add_layer_norm", "block"])
def test_hooks_that_give_something_else_back_are_refused(name):
    """Of another size, another type or on the host: before anything runs."""
    show("hooks that give something else", name)
    call, inputs = layer_calls(torch.bfloat16)[name]
    shapes = {tuple(t.shape) for t in inputs}
    for wrong in (lambda t: t[:-1], lambda t: t.cpu(), lambda t: t.to(torch.int16), lambda t: torch.cat((t, t))[::2]):
        leaves = [t.clone().requires_grad_(True) for t in inputs]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t if tuple(t.shape) in shapes else wrong(t)):
            out = call(*leaves)
        out = out if isinstance(out, tuple) else (out,)
        with pytest.raises(RuntimeError, match="what the forward pass left"):
            torch.autograd.grad(out, leaves, [torch.ones_like(t) for t in out])


def test_hooks_that_give_another_weight_back_are_refused():
    show("hooks that give another weight")
    call, inputs = layer_calls(torch.bfloat16)["layer_norm"]
    for wrong in (lambda t: t[:-1], lambda t: t.float(), lambda t: t.half(), lambda t: t.cpu()):
        leaves = [t.clone().requires_grad_(True) for t in inputs]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: wrong(t) if t.shape == (40,) else t):
            y = call(*leaves)
        with pytest.raises(RuntimeError, match="weight must"):
            torch.autograd.grad(y, leaves, torch.ones_like(y))


# ---------------------------------------------------------------- very wide rows

def test_parameter_gradients_of_very_wide_rows():
    """2^26 and some columns, where a workgroup for every 32 of them is more than a launch may have.  Rows of as many 1 as -1 have the mean 0
    and the spread 1 exactly, so that hat is x / sqrt(1 + eps) to 4 units of the last place, and bfloat16 sums of two are rounded once."""
    show("very wide rows")
    width = (1 << 26) + 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.ones((2, width), device="cuda", dtype=torch.bfloat16)
    x[0, 1::2] = -1.0
    x[1, :width // 2] = -1.0
    w, b = (torch.randn(width, device="cuda", generator=gen).to(torch.bfloat16).requires_grad_(True) for _ in range(2))
    dy = torch.randn((2, width), device="cuda", generator=gen).to(torch.bfloat16)
    y = layers.layer_norm(x, w, b)
    dw, db = torch.autograd.grad(y, [w, b], dy)
    u, e = 2.0 ** -8, 2.0 ** -24
    hat = x.double() / (1 + 1e-5) ** 0.5
    assert ((y.detach().double() - hat * w.detach().double() - b.detach().double()).abs()
            <= (u + 8 * e) * (w.detach().double().abs() + b.detach().double().abs())).all()
    assert torch.equal(db, (dy[0].float() + dy[1].float()).to(torch.bfloat16))
    terms = dy.double() * hat
    assert ((dw.double() - terms.sum(0)).abs() <= u * terms.sum(0).abs() + 8 * e * terms.abs().sum(0)).all()


# ---------------------------------------------------------------- views that count as negative

def test_views_whose_sign_is_not_in_memory():
    """torch marks some views as negative, such as the imaginary part of a conjugate, in place of writing them."""
    show("negative views")
    for dtype in TYPES:
        for name, (call, inputs) in layer_calls(dtype).items():
            grads = [torch.randn_like(t) for t in (lambda o: o if isinstance(o, tuple) else (o,))(call(*inputs))]
            found = []
            for view in (lambda t: torch._neg_view(-t), lambda t: t):
                leaves = [view(t).requires_grad_(True) for t in inputs]
                out = call(*leaves)
                out = out if isinstance(out, tuple) else (out,)
                found.append([*out, *torch.autograd.grad(out, leaves, [view(g) for g in grads])])
            assert all(torch.equal(a, b) for a, b in zip(*found)), (name, dtype)
    z = torch.randn((30, 1), device="cuda", dtype=torch.complex64)
    assert torch.equal(layers.dropout(z.conj().imag, 0.5, 1), layers.dropout(-z.imag, 0.5, 1))


# ---------------------------------------------------------------- more rows than workgroups

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(70001, 8), (40003, 33), (33001, 64), (5001, 500), (4101, 600), (2501, 1001), (1700, 2050), (600, 8192), (530, 8200)])
def test_norms_of_more_rows_than_workgroups(rows, width, dtype):
    """Each goes on to further rows, asked for while the ones before are worked on; rows in a team's lanes, in a workgroup and read again."""
    import test_layers as t
    show("many rows", rows, width, dtype)
    x, r, dy, ds = (t.normal((rows, width), dtype, 200 + i, 1.3, 0.4) for i in range(4))
    w, b = t.normal((width,), dtype, 204, 0.2, 1.0), t.normal((width,), dtype, 205)
    t.check_norm(x, w, b, dy)
    t.check_add_norm(x, r, w, b, dy, ds, 0.25)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,hidden,out", [(70, 64, 128, 64), (70, 60, 100, 33), (70, 64, 256, 64), (70, 300, 264, 136), (300, 250, 333, 131), (4096, 256, 1024, 256)])
def test_what_is_not_finite_stays_in_its_row(rows, width, hidden, out, dtype):
    """An infinity or NaN in a row of x or dy is in that row's result and gradient, and in no other's; beside it the bits are the same."""
    show("not finite", rows, width, hidden, out, dtype)
    torch.manual_seed(0)
    x, dy = torch.randn((rows, width), device="cuda").to(dtype), torch.randn((rows, out), device="cuda").to(dtype)
    w = [(torch.randn(shape, device="cuda") * shape[1] ** -0.5).to(dtype) for shape in ((hidden, width), (hidden, width), (out, hidden))]

    def passes(x, dy):
        leaf = x.clone().requires_grad_(True)
        y = layers.gated_ff(leaf, *w)
        return y.detach(), torch.autograd.grad(y, leaf, dy)[0]

    want = passes(x, dy)
    for bad in (float("nan"), float("inf"), float("-inf")):
        spoilt, grad = x.clone(), dy.clone()
        spoilt[[0, 37], [width - 1, 5]] = bad
        grad[[1, rows - 1], [0, out - 1]] = bad
        others = torch.ones(rows, dtype=torch.bool, device="cuda")
        others[[0, 37]] = False
        y, dx = passes(spoilt, dy)
        assert torch.equal(y[others], want[0][others]) and torch.equal(dx[others], want[1][others])
        assert not torch.isfinite(y[[0, 37]]).any()
        y, dx = passes(x, grad)
        others[:] = True
        others[[1, rows - 1]] = False
        assert torch.equal(y, want[0]) and torch.equal(dx[others], want[1][others])
        assert not torch.isfinite(dx[[1, rows - 1]]).any()


# ---------------------------------------------------------------- offsets beyond 32 bits

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_rows_far_apart(dtype):
    """2^30 elements from row to row of inputs, weights and gradients: the same bits as of packed ones."""
    show("rows far apart", dtype)
    torch.manual_seed(0)
    rows, apart = 6, 1 << 30
    store = torch.empty((rows - 1) * apart + 8192, dtype=dtype, device="cuda")

    def far(t, at):
        view = store.as_strided(t.shape, (apart, 1), at)
        view.copy_(t)
        return view

    def same(call, inputs, grad):
        found = []
        for place in (far, lambda t, at: t):
            grads = [place(g, 700 * (len(inputs) + i)) for i, g in enumerate(grad)]
            leaves = [place(t, 700 * i).detach().requires_grad_(True) if t.dim() == 2 else t.requires_grad_(True) for i, t in enumerate(inputs)]
            out = call(*leaves)
            out = out if isinstance(out, tuple) else (out,)
            found.append([*out, *torch.autograd.grad(out, leaves, grads)])
        assert all(torch.equal(a, b) for a, b in zip(*found))

    def normal(*shape):
        return torch.randn(shape, device="cuda").to(dtype)

    same(lambda x, w, b: layers.layer_norm(x, w, b), [normal(rows, 600), normal(600), normal(600)], [normal(rows, 600)])
    same(lambda x, r: layers.add_layer_norm(x, r, p=0.25, seed=1), [normal(rows, 600), normal(rows, 600)], [normal(rows, 600)] * 2)
    same(lambda x, r: layers.dropout(x, 0.25, 1, residual=r), [normal(rows, 600), normal(rows, 600)], [normal(rows, 600)])
    for width in (64, 600):
        same(layers.gated_ff, [normal(rows, width), normal(6, width), normal(6, width), normal(rows, 6)], [normal(rows, 6)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_norms_of_more_than_2_to_the_31_elements(dtype):
    """The first and the last rows give what they give alone, and the parameters' gradients are sums over all."""
    show("many elements", dtype)
    rows, width = (1 << 20) + 77, 2056
    x = torch.empty((rows, width), dtype=dtype, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(0))
    w = torch.randn(width, device="cuda").to(dtype).requires_grad_(True)
    x.requires_grad_(True)
    y = layers.layer_norm(x, w, None)
    dx, dw = torch.autograd.grad(y, [x, w], x.detach())
    for part in (slice(0, 100), slice(rows - 100, rows)):
        alone = x.detach()[part].clone().requires_grad_(True)
        one = layers.layer_norm(alone, w, None)
        assert torch.equal(one, y[part]) and torch.equal(torch.autograd.grad(one, alone, alone.detach())[0], dx[part])
    want = torch.zeros(width, dtype=torch.float64, device="cuda")
    for part in x.detach().split(1 << 16):
        s = part.double()
        want += (s * torch.nn.functional.layer_norm(s, (width,))).sum(0)
    assert ((dw.double() - want).abs() <= (UNIT[dtype] + 2.0 ** -10) * want).all()               # sums of squares: 2^-24 a term of the 1024 that a lane adds, and more
    keep = layers.dropout(x.detach(), 0.5, 1, residual=x.detach())
    assert torch.equal(keep[-100:, :8], torch.where(layers.dropout(torch.ones((rows, 8), device="cuda", dtype=dtype), 0.5, 1)[-100:] > 0, 3.0, 1.0).to(dtype) * x.detach()[-100:, :8])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_a_block_of_more_than_2_to_the_31_hidden_values(dtype):
    """The first and the last rows against 64 bits with their bounds, the weights' gradients, sums over 2^20 rows, to a hundredth of their size."""
    import test_layers_tiles as t
    show("many hidden values", dtype)
    rows, width, hidden, out = (1 << 20) + 77, 40, 2056, 24
    gen = torch.Generator("cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen).mul_(scale)

    x, w, dy = normal(rows, width), [normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5),
                                     normal(out, hidden, scale=hidden ** -0.5)], normal(rows, out)
    y, dx, *dw = t.passes([x, *w, dy], "silu")
    sums = [torch.zeros(v.shape, dtype=torch.float64, device="cuda") for v in w]
    wide = [v.double() for v in w]
    for first in range(0, rows, 1 << 16):
        part = slice(first, min(rows, first + (1 << 16)))
        found = t.definition(x[part].double(), *wide, dy[part].double(), "silu", dtype)
        if first == 0 or part.stop == rows:
            for got, (value, bound), name in zip((y[part], dx[part]), found, ("y", "dx")):
                t.assert_within(got, value.cpu(), bound.cpu(), name)
        for s, (value, _) in zip(sums, found[2:]):
            s += value
    for got, s in zip(dw, sums):
        assert (got.double() - s).norm() <= 1e-2 * s.norm()
