"""Norm, product and rows in 8 bits at the edges of what they take: offsets beyond 32 bits, the widest rows, numbers that are none, graphs
that are captured and replayed beside others, calls from several threads."""
import gc
import threading

import pytest
import torch

import linear_reference as lin
from layer_reference import UNIT
from paper_2106_16064_amd import layers
from test_linear import check, inputs
from test_linear_8bit import check as check_8bit
from test_rms_norm import gradient

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def show(*case):
    print("[case]", *case, flush=True)


def normal(shape, dtype, seed, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(seed)).mul_(scale)


def within(got, want, bound, name):
    assert ((got.double() - want).abs() <= bound).all(), name


# ---------------------------------------------------------------- offsets beyond 32 bits

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,apart", [(6, 1 << 30), (70, 1 << 25)])
def test_rows_far_apart(rows, apart, dtype):
    """Inputs, weights and gradients whose rows lie 2^30 or 2^25 elements from each other: the same bits as of packed ones."""
    show("rows far apart", rows, dtype)
    store = torch.empty((rows - 1) * apart + 16384, dtype=dtype, device="cuda")

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

    n = lambda *shape: normal(shape, dtype, len(shape) + shape[-1])  # noqa: E731
    same(lambda x, w: layers.rms_norm(x, w), [n(rows, 600), n(600)], [n(rows, 600)])
    same(lambda x, r: layers.add_rms_norm(x, r, p=0.25, seed=1), [n(rows, 600), n(rows, 600)], [n(rows, 600)] * 2)
    for width in (64, 600):
        for keep in (False, True):
            same(lambda x, w, r: layers.linear(x, w, None, "gelu", r, keep), [n(rows, width), n(6, width), n(rows, 6)], [n(rows, 6)])
    x, r = n(rows, 600), normal((rows, 600), dtype, 5)
    for f in (layers.quantise, lambda t: layers.quantise(t, "int8"), layers.rms_norm_8bit, lambda t: layers.add_rms_norm_8bit(t, far(r, 700))[0]):
        a, b = f(far(x, 0)), f(x)
        assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)


@pytest.mark.gpu
def test_values_far_apart():
    """Rows of values as far apart as products read them in place, 8 MiB, and more than 2^31 bytes in all; and farther, where they are copied."""
    show("values far apart")
    x8, w8 = layers.quantise(normal((300, 400), torch.bfloat16, 1)), layers.quantise(normal((130, 400), torch.bfloat16, 2))
    want = layers.linear_8bit(x8, w8, None, "silu")
    store = torch.empty(300 * (1 << 23) + 1024, dtype=torch.uint8, device="cuda")
    for apart in ((1 << 23) - 16, 1 << 23):
        def far(t, at):
            view = store.as_strided(t.values.shape, (apart, 1), at)
            view.copy_(t.values.view(torch.uint8))
            return layers.Rows8(view.view(torch.float8_e4m3fn), t.scales, t.width)
        a, b = far(x8, 0), far(w8, 512)
        assert torch.equal(layers.linear_8bit(a, b, None, "silu"), want)
        assert torch.equal(layers.dequantise(a), layers.dequantise(x8))
        few = layers.Rows8(a.values[:5], x8.scales[:, :5], 400)
        assert torch.equal(layers.linear_8bit(few, b), layers.linear_8bit(layers.Rows8(x8.values[:5], x8.scales[:, :5], 400), w8))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_norms_of_more_than_2_to_the_31_elements(dtype):
    """The first and the last rows give what they give alone, and the weight's gradient is the sum over all."""
    show("norms of many elements", dtype)
    rows, width = (1 << 20) + 77, 2056
    x, r = normal((rows, width), dtype, 0).requires_grad_(True), normal((rows, width), dtype, 1)
    w = normal((width,), dtype, 2).requires_grad_(True)
    y, s = layers.add_rms_norm(x, r, w)
    dx, dw = torch.autograd.grad([y, s], [x, w], [r, x.detach()])
    ends = (slice(0, 100), slice(rows - 100, rows))
    for part in ends:
        alone, beside = x.detach()[part].clone().requires_grad_(True), r[part].clone()
        one = layers.add_rms_norm(alone, beside, w)
        assert torch.equal(one[0], y[part]) and torch.equal(one[1], s[part])
        assert torch.equal(torch.autograd.grad(one, alone, [beside, alone.detach()])[0], dx[part])
    want = torch.zeros(width, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for first in range(0, rows, 1 << 16):
        part = slice(first, min(rows, first + (1 << 16)))
        sum_ = x.detach()[part].double() + r[part].double()
        terms = r[part].double() * sum_ / torch.sqrt((sum_ * sum_).mean(1, keepdim=True) + 1e-5)
        want += terms.sum(0)
        size += terms.abs().sum(0)
    # of the 768 workgroups a lane adds 1366 terms, one after the other, 2^-13.5 of their magnitudes, and a mean of 2056 squares moves its row by 2^-14
    assert ((dw.double() - want).abs() <= UNIT[dtype] * want.abs() + 2.0 ** -12 * size).all()
    with torch.no_grad():
        assert torch.equal(layers.add_rms_norm(x, r, p=0.5, seed=3)[1][-100:], layers.dropout(x, 0.5, 3, residual=r)[-100:])
        eight = layers.add_rms_norm_8bit(x, r, w)[0]
        for part in ends:
            one = layers.add_rms_norm_8bit(x[part].clone(), r[part].clone(), w)[0]
            assert torch.equal(eight.values[part].view(torch.uint8), one.values.view(torch.uint8)) and torch.equal(eight.scales[:, part], one.scales)
        del y, s, dx, eight
        for kind in ("e4m3", "int8"):
            whole = layers.quantise(x, kind)
            back = layers.dequantise(whole, dtype)
            for part in ends:
                one = layers.quantise(x[part].clone(), kind)
                assert torch.equal(whole.values[part].view(torch.uint8), one.values.view(torch.uint8)) and torch.equal(whole.scales[:, part], one.scales)
                assert torch.equal(back[part], layers.dequantise(one, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_the_norms_weight_gradient_has_the_rows_at_both_ends_and_beyond_2_to_the_31(dtype):
    """dy is zero but for some rows at the ends and around the 2^31st element, so that each of them counts: each adds its own term, and zeros, in
    some thousand sums."""
    show("rows that count", dtype)
    rows, width = (1 << 20) + 77, 2056
    x, dy = normal((rows, width), dtype, 0), torch.zeros((rows, width), dtype=dtype, device="cuda")
    some = torch.cat([torch.arange(5), (1 << 31) // width + torch.arange(-3, 4), torch.arange(rows - 80, rows)]).cuda()
    dy[some] = normal((len(some), width), dtype, 1)
    w = normal((width,), dtype, 2).requires_grad_(True)
    dw, = torch.autograd.grad(layers.rms_norm(x, w), w, dy)
    S, G = x[some].double(), dy[some].double()
    value, off = (t.cuda() for t in gradient(S.cpu(), torch.zeros_like(S.cpu()), w.detach().double().cpu(), G.cpu(), 1e-5)[2:])
    within(dw, value, off * (1 + UNIT[dtype]) + UNIT[dtype] * value.abs(), "dw")

@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("width,out", [(40, 2056), (2056, 24)])
def test_products_of_more_than_2_to_the_31_elements(width, out, dtype, keep):
    """The first and the last rows against 64 bits with their bounds, the weight's gradient, a sum over 2^20 rows, to a hundredth of its size:
    dz is rounded by 2^-8 of itself, slopes to steps of 1/112 (0.0026 in the mean, beside a slope of about 0.6), with any sign."""
    show("products of many elements", width, out, dtype, keep)
    rows = (1 << 20) + 77
    x, w, dy, r = normal((rows, width), dtype, 0), normal((out, width), dtype, 1, width ** -0.5), normal((rows, out), dtype, 2), normal((rows, out), dtype, 3)
    leaves = [x.requires_grad_(True), w.requires_grad_(True)]
    y = layers.linear(*leaves, None, "gelu", r, keep)
    dx, dw = torch.autograd.grad(y, leaves, dy)
    kept = layers.dequantise(layers.quantise(x.detach(), "int8"), dtype) if keep else x.detach()
    w = w.detach().double()
    total = torch.zeros((out, width), dtype=torch.float64, device="cuda")
    for first in range(0, rows, 1 << 15):
        part = slice(first, min(rows, first + (1 << 15)))
        X, G = x.detach()[part].double(), dy[part].double()
        (want, bound), (z, off) = lin.forward(X, w, None, "gelu", r[part].double(), dtype)
        if first == 0 or part.stop == rows:
            within(y.detach()[part], want, bound, "y")
            value, bound = lin.backward(kept[part].double(), w, z, off, "gelu", G, dtype, dtype, keep)[0]
            within(dx[part], value, bound, "dx")
        total += (G * lin.slope("gelu", z)).t() @ kept[part].double()
    assert (dw.double() - total).norm() <= 1e-2 * total.norm()


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, 72), (torch.float32, 64)], ids=str)
def test_narrow_products_of_more_than_2_to_the_31_elements(dtype, out, keep):
    show("narrow products of many elements", dtype, keep)
    rows, width = (1 << 25) + 77, 64
    x, w, dy, r = normal((rows, width), dtype, 0), normal((out, width), dtype, 1, 0.125), normal((rows, out), dtype, 2), normal((rows, out), dtype, 3)
    leaves = [x.requires_grad_(True), w.requires_grad_(True)]
    y = layers.linear(*leaves, None, "silu", r, keep)
    dx, dw = torch.autograd.grad(y, leaves, dy)
    for part in (slice(0, 100), slice(rows - 100, rows)):                   # of narrow rows one kernel takes any number
        alone = x.detach()[part].clone().requires_grad_(True)
        one = layers.linear(alone, leaves[1], None, "silu", r[part].clone(), keep)
        assert torch.equal(one, y[part]) and torch.equal(torch.autograd.grad(one, alone, dy[part].clone())[0], dx[part])
    total = torch.zeros((out, width), dtype=torch.float64, device="cuda")
    for first in range(0, rows, 1 << 20):
        part = slice(first, min(rows, first + (1 << 20)))
        X = x.detach()[part].double()
        read = layers.dequantise(layers.quantise(x.detach()[part], "int8"), dtype).double() if keep else X
        total += (dy[part].double() * lin.slope("silu", X @ w.detach().double().t())).t() @ read
    assert (dw.double() - total).norm() <= 1e-2 * total.norm()              # as of the wide ones


@pytest.mark.gpu
@pytest.mark.parametrize("width,out", [(40, 2056), (2056, 24)])
def test_8_bit_products_of_more_than_2_to_the_31_elements(width, out):
    show("8-bit products of many elements", width, out)
    rows = (1 << 20) + 77
    x8, w8, r = layers.quantise(normal((rows, width), torch.float32, 0)), layers.quantise(normal((out, width), torch.float32, 1)), normal((rows, out), torch.bfloat16, 2)
    y = layers.linear_8bit(x8, w8, None, "gelu", r)

    def scales(t):
        return 2.0 ** (t.scales.transpose(0, 1).reshape(t.scales.shape[1], -1)[:, :-(-width // 32)].double() - 127)

    W = layers.dequantise(w8).double()
    for part in (slice(0, 5000), slice(rows - 5000, rows)):
        some = layers.Rows8(x8.values[part], x8.scales[:, part], width)
        X = layers.dequantise(some).double()
        want, bound = lin.forward(X, W, None, "gelu", r[part].double(), torch.bfloat16, lin.cut_off_in_8bit(X, W, scales(some), scales(w8)))[0]
        within(y[part], want, bound, "y")


# ---------------------------------------------------------------- the widest rows

@pytest.mark.gpu
def test_norm_of_very_wide_rows():
    """2^26 and some columns of 1 and -1, whose mean square is 1 exactly, so that hat is x / sqrt(1 + eps) to 4 units of the last place; bfloat16
    sums of two are rounded once."""
    show("very wide rows")
    width = (1 << 26) + 16
    x = torch.ones((2, width), device="cuda", dtype=torch.bfloat16)
    x[0, 1::2] = -1.0
    x[1, :width // 2] = -1.0
    w, dy = normal((width,), torch.bfloat16, 0).requires_grad_(True), normal((2, width), torch.bfloat16, 1)
    y = layers.rms_norm(x, w)
    dw, = torch.autograd.grad(y, [w], dy)
    u, e = 2.0 ** -8, 2.0 ** -24
    hat = x.double() / (1 + 1e-5) ** 0.5
    want = hat * w.detach().double()
    within(y.detach(), want, (u + 8 * e) * want.abs(), "y")
    terms = dy.double() * hat
    within(dw, terms.sum(0), u * terms.sum(0).abs() + 8 * e * terms.abs().sum(0), "dw")
    with torch.no_grad():
        eight = layers.rms_norm_8bit(x, w)
    scale = 2.0 ** (eight.scales.transpose(0, 1).reshape(2, -1)[:, :-(-width // 32)].double() - 127)
    per = scale.repeat_interleave(32, 1)[:, :width]
    within(layers.dequantise(eight), want, torch.maximum((2.0 ** -4 + 8 * e) * want.abs(), 2.0 ** -10 * per + 8 * e * want.abs()), "y in 8 bits")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows", [2, 70])
@pytest.mark.parametrize("width,out", [((1 << 22) - 8, 3), (3, (1 << 22) - 8)])
def test_widest_products(width, out, rows, dtype):
    """Of -1, 0 and 1, whose sums are exact in 32 bits: the results are those of 64 bits, rounded once."""
    show("widest products", width, out, rows, dtype)

    def digits(shape, seed):
        return torch.randint(-1, 2, shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).to(dtype)

    x, w, dy = digits((rows, width), 0).requires_grad_(True), digits((out, width), 1).requires_grad_(True), digits((rows, out), 2)
    b = digits((out,), 3).requires_grad_(True)
    X, W, G = x.detach().double(), w.detach().double(), dy.double()
    y = layers.linear(x, w, b)
    assert torch.equal(y, (X @ W.t() + b.detach().double()).to(dtype))
    got = torch.autograd.grad(y, [x, w, b], dy)
    assert all(torch.equal(a, v.to(dtype)) for a, v in zip(got, (G @ W, G.t() @ X, G.sum(0))))
    kept = layers.linear(x, w, b, keep_8bit=True)                            # a block's scale is 2^-6, and 64 of it are 1
    assert torch.equal(kept, y) and all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(kept, [x, w, b], dy), got))
    with torch.no_grad():
        assert torch.equal(layers.linear_8bit(layers.quantise(x), layers.quantise(w), b, dtype=dtype), y)


# ---------------------------------------------------------------- deep sums

@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,out", [(2800, 8300, 2560), (200, 4096, 5000), (1, 20000, 300), (16, 4096, 1000), (33, 4096, 130)])
def test_deep_sums_in_8_bits(rows, width, out):
    show("deep sums in 8 bits", rows, width, out)
    check_8bit(rows, width, out, torch.bfloat16, "silu", 300, at="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,width,out", [
    (torch.bfloat16, 12000, 1500, 2000), (torch.float16, 10300, 1040, 1024), (torch.bfloat16, 8200, 1024, 4096), (torch.bfloat16, 50000, 301, 777),
    (torch.bfloat16, 200, 4096, 5000), (torch.float16, 2800, 4104, 2560), (torch.bfloat16, 16, 16384, 520), (torch.float32, 50000, 64, 64), (torch.float32, 30000, 33, 128), (torch.float32, 40000, 33, 70), (torch.float32, 20001, 129, 130), (torch.float32, 8200, 128, 512),
    (torch.float32, 4100, 2048, 2050), (torch.float32, 3000, 31, 33), (torch.float32, 1000, 300, 200)], ids=str)
def test_deep_sums(dtype, rows, width, out):
    """Weights' gradients that are split to fill the GPU, with tiles of each size, few and many splits and results; of float their bias's beside them."""
    show("deep sums", dtype, rows, width, out)
    for seed, (kind, params, keep) in enumerate([(None, dtype, False), (None, torch.float32, True), ("gelu", dtype, True)]):
        check(inputs(rows, width, out, dtype, params, 200 + 10 * seed), kind, keep, at="cuda")


# ---------------------------------------------------------------- numbers that are none

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(70, 64, 72), (70, 200, 300), (9, 520, 40)])
@pytest.mark.parametrize("keep", [False, True])
def test_nan_reaches_all_that_depends_on_it(keep, rows, width, out, dtype):
    """A NaN of x: its row of y and of dx, and all of dweight and dbias, which are sums over the rows; other rows keep their bits."""
    show("nan", rows, width, out, dtype, keep)
    x, w, b, dy = normal((rows, width), dtype, 0), normal((out, width), dtype, 1, width ** -0.5), normal((out,), dtype, 2), normal((rows, out), dtype, 3)
    found = []
    for bad in (False, True):
        t = x.clone()
        if bad:
            t[rows // 2, 37] = float("nan")
        leaves = [t.requires_grad_(True), w.clone().requires_grad_(True), b.clone().requires_grad_(True)]
        for kind in ("silu", "gelu"):
            y = layers.linear(*leaves, kind, keep_8bit=keep)
            found.append([y.detach(), *torch.autograd.grad(y, leaves, dy)])
    others = [i for i in range(rows) if i != rows // 2]
    for clean, dirty in zip(found[:2], found[2:]):
        for a, c in zip(clean[:2], dirty[:2]):
            assert torch.equal(a[others], c[others]) and torch.isnan(c[rows // 2]).all()
        assert torch.isnan(dirty[2]).all() and torch.isnan(dirty[3]).all()


# ---------------------------------------------------------------- graphs and threads

@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
def test_two_captured_graphs_run_beside_each_other(keep):
    """Each has workspaces of its own: replayed on two streams at once, many times, both give what they give alone."""
    show("two graphs", keep)
    steps, graphs, results, wants = [], [], [], []
    for seed, (rows, width, out) in enumerate([(30, 4100, 70), (200, 2050, 130)]):
        x, w, b, dy = (normal(shape, torch.bfloat16, 10 * seed + i) for i, shape in enumerate([(rows, width), (out, width), (out,), (rows, out)]))
        leaves = [t.requires_grad_(True) for t in (x, w, b)]

        def step(leaves=leaves, dy=dy):
            y = layers.linear(*leaves, "gelu", keep_8bit=keep)
            with torch.no_grad():
                n = layers.linear_8bit(layers.rms_norm_8bit(leaves[0]), layers.quantise(leaves[1]))
            return [y.detach(), n, *torch.autograd.grad(y, leaves, dy)]

        steps.append(step)
        wants.append(step())
    torch.cuda.synchronize()
    for step in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(step())
        graphs.append(graph)
    sides = [torch.cuda.Stream() for _ in graphs]
    for turn in range(10):
        for got in results:
            for t in got:
                t.zero_()
        torch.cuda.synchronize()
        for graph, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(results, wants):
            assert all(torch.equal(a, c) for a, c in zip(got, want)), turn


@pytest.mark.gpu
def test_a_gradient_is_not_captured_while_an_eager_graph_holds_the_leaf():
    """Torch would send it to the default stream, which takes part in no capture, and end the process: the call is refused, and the capture goes on."""
    show("capture beside an eager graph")
    calls = {
        "rms_norm": lambda t: layers.rms_norm(t),
        "linear": lambda t: layers.linear(t, weight, None, "gelu"),
        "layer_norm": lambda t: layers.layer_norm(t),
    }
    weight = normal((40, 200), torch.float32, 1)
    for name, call in calls.items():
        leaf = normal((30, 200), torch.float32, 2).requires_grad_(True)
        held = layers.rms_norm(leaf)                                         # on the default stream
        graph, dy = torch.cuda.CUDAGraph(), torch.ones_like(call(leaf.detach()))
        with torch.cuda.graph(graph):
            y = call(leaf)
            with pytest.raises(RuntimeError, match="cannot be captured"):
                torch.autograd.grad(y, leaf, dy)
            y = y.detach()
        del held
        gc.collect()
        again = torch.cuda.CUDAGraph()
        with torch.cuda.graph(again):
            y = call(leaf)
            g, = torch.autograd.grad(y, leaf, dy)
            y = y.detach()
        want = call(leaf)
        slope, = torch.autograd.grad(want, leaf, dy)
        for _ in range(3):
            again.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(g, slope), name


@pytest.mark.gpu
def test_calls_from_several_threads():
    show("threads")
    inputs = [[normal(shape, torch.bfloat16, 10 * i + j) for j, shape in enumerate([(33 + i, 2050), (70, 2050), (33 + i, 70)])] for i in range(4)]

    def work(t):
        leaves = [v.clone().requires_grad_(True) for v in t[:2]]
        y = layers.linear(layers.rms_norm(leaves[0]), leaves[1], None, "silu", t[2], True)
        with torch.no_grad():
            n = layers.linear_8bit(layers.rms_norm_8bit(t[0]), layers.quantise(t[1]))
        return [y.detach(), n, *torch.autograd.grad(y, leaves, t[2])]

    wants = [work(t) for t in inputs]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for turn in range(20):
                got = work(inputs[i])
                side.synchronize()
                if not all(torch.equal(a, c) for a, c in zip(got, wants[i])):
                    wrong.append((i, turn))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
