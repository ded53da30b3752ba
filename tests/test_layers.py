"""Layer norm, dropout and the gated feed-forward block on the GPU against their definitions in 64 bits.

Bounds, element by element.  A result is rounded once: u |y| with u = 2^-24, 2^-8, 2^-11 for float32, bfloat16, float16.  A sum
of n products in 32 bits in any order is off by at most (n + 4) 2^-24 times the sum of the magnitudes.  What a kernel rounds in
between (the hidden values of the feed-forward block, the sum that the norm's backward pass reads) adds u times its magnitude,
carried through the products behind it.  exp, erf and square roots of 32 bits: 4 units in the last place."""
import pytest
import torch

import layer_reference as ref
from layer_reference import EPS32, TINY, UNIT, assert_within
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-5


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, dtype, seed, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float64) * scale + shift).to(dtype)


def host(t):
    return None if t is None else t.detach().double().cpu()


def show(*case):
    print("[case]", *case, flush=True)


# ---------------------------------------------------------------- layer norm

def norm_bound(s, weight, bias, u, eps=EPS):
    """Of y: the mean is off by (n + 4) e mean|s|, and what is left of s by that and by its own rounding; relative errors of the
    spread, the square root and the last two steps."""
    n = s.shape[1]
    mean = s.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + eps)
    hat = (s - mean).abs() * rstd
    shift = (n + 4) * EPS32 * s.abs().mean(1, keepdim=True) + 2 * EPS32 * (s.abs() + mean.abs())
    w = weight.abs() if weight is not None else 1.0
    b = bias.abs() if bias is not None else 0.0
    # the spread is off by (n + 8) e relative, plus the square of the mean's error
    spread = (n + 8) * EPS32 + (shift * rstd) ** 2
    return (shift * rstd + hat * spread) * w + (u + 4 * EPS32) * (hat * w + b)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 4096), (3, 2), (5, 3), (64, 7), (33, 8), (1025, 31), (257, 32), (63, 33), (7, 64), (9, 65),
                                        (130, 127), (65, 128), (6, 256), (5, 257), (4, 500), (3, 512), (3, 513), (4, 1000), (5, 1001),
                                        (2, 2048), (2, 2050), (2, 4095), (3, 8192), (2, 8193), (1, 20000), (1, 70001)])
def test_layer_norm(rows, width, dtype):
    show("layer_norm", rows, width, dtype)
    for params in {dtype, torch.float32}:
        x = normal((rows, width), dtype, 1, 2.0, 0.7)
        w, b = normal((width,), params, 2, 0.2, 1.0), normal((width,), params, 3, 0.3)
        dy = normal((rows, width), dtype, 4)
        dx_, dw_, db_ = check_norm(x, w, b, dy)
        assert dx_.dtype == dtype and dw_.dtype == params and db_.dtype == params


def check_norm(x, w, b, dy, eps=EPS, place=lambda t: t.cuda()):
    """Forward and backward of tensors on the host; `place` puts those of two axes on the GPU.  Returns the gradients."""
    u, up = UNIT[x.dtype], UNIT[(w if w is not None else x).dtype]
    leaves = [place(x).requires_grad_(True), *(None if t is None else t.cuda().requires_grad_(True) for t in (w, b))]
    y = layers.layer_norm(*leaves, eps=eps)
    X, W, B, G = host(x), host(w), host(b), host(dy)
    want = ref.norm(X, W, B, eps)
    assert_within(y, want, norm_bound(X, W, B, u, eps) + TINY[x.dtype], "y")
    with torch.no_grad():
        assert torch.equal(layers.layer_norm(*leaves, eps=eps), y)                    # without a graph: the same bits
    grads = torch.autograd.grad(y, [t for t in leaves if t is not None], place(dy))
    check_norm_gradient(X, W, G, grads[0], *([g for g in grads[1:]] + [None, None])[:2], u, up, eps, slack=0.0)
    return grads


def check_norm_gradient(S, W, G, ds, dw, db, u, up, eps, slack, extra=None):
    """`slack`: by how much, relative to its magnitude, the kernel's s may differ from S."""
    rows, n = S.shape
    want, want_w, want_b = ref.norm_gradient(S, W, G, eps)
    mean = S.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((S - mean) ** 2).mean(1, keepdim=True) + eps)
    hat = (S - mean) * rstd
    dhat = (G if W is None else G * W).abs()
    # hat as the kernel sees it is off by this much
    off = ((n + 8) * EPS32 * S.abs().mean(1, keepdim=True) + (slack + 2 * EPS32) * (S.abs() + mean.abs())) * rstd + (n + 8) * EPS32 * hat.abs()
    b = (dhat * hat.abs()).mean(1, keepdim=True)
    bound = (dhat * 4 * EPS32 + (n + 8) * EPS32 * (dhat.mean(1, keepdim=True) + hat.abs() * b) + off * b
             + (hat.abs() + off) * (dhat * off).mean(1, keepdim=True)) * rstd
    bound = bound + ((n + 8) * EPS32 + (off ** 2)) * (dhat + dhat.mean(1, keepdim=True) + hat.abs() * b) * rstd
    if extra is not None:
        want = want + extra
        bound = bound + 2 * EPS32 * extra.abs()
    assert_within(ds, want, bound + u * want.abs() + TINY[ds.dtype], "ds")
    if dw is not None:
        assert_within(dw, want_w, (rows + 8) * EPS32 * (G * hat).abs().sum(0) + (G.abs() * off).sum(0) + up * want_w.abs() + TINY[dw.dtype], "dweight")
    if db is not None:
        assert_within(db, want_b, (rows + 8) * EPS32 * G.abs().sum(0) + up * want_b.abs() + TINY[db.dtype], "dbias")
    return want, bound


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(4, 24), (3, 1000), (70, 40)])
def test_layer_norm_without_parameters(rows, width, dtype):
    show("no parameters", rows, width, dtype)
    x, dy = normal((rows, width), dtype, 5, 1.5, -1.0), normal((rows, width), dtype, 6)
    w, b = normal((width,), dtype, 7, 0.2, 1.0), normal((width,), dtype, 8)
    check_norm(x, None, None, dy)
    check_norm(x, w, None, dy)
    leaf, bias = x.cuda().requires_grad_(True), b.cuda().requires_grad_(True)
    y = layers.layer_norm(leaf, None, bias)
    assert_within(y, ref.norm(host(x), None, host(b), EPS), norm_bound(host(x), None, host(b), UNIT[dtype]) + TINY[dtype], "y")
    assert torch.autograd.grad(y, bias, dy.cuda())[0].shape == (width,)


@pytest.mark.parametrize("rows,width", [(1, 40), (4100, 48), (20000, 5), (9000, 260)])
def test_parameter_gradients_over_many_rows(rows, width):
    show("many rows", rows, width)
    for dtype in (torch.float32, torch.bfloat16):
        check_norm(normal((rows, width), dtype, 9), normal((width,), torch.float32, 10, 0.1, 1.0), normal((width,), torch.float32, 11),
                   normal((rows, width), dtype, 12))


def test_rows_that_leave_nothing():
    """Constant rows have no spread, a large mean hides the spread behind it, and a row with an infinity stays alone."""
    show("constant rows")
    x = normal((6, 130), torch.float32, 13)
    x[1] = 3.25
    x[2] = 0.0
    x[3] = x[3] * 1e-3 + 1000.0
    check_norm(x, normal((130,), torch.float32, 14, 0.1, 1.0), normal((130,), torch.float32, 15), normal((6, 130), torch.float32, 16))
    for bad in (float("inf"), float("-inf"), float("nan")):
        z = normal((6, 130), torch.float32, 13)
        z[4, 77] = bad
        y = layers.layer_norm(z.cuda()).cpu()
        assert torch.isnan(y[4]).all() and torch.isfinite(y[[0, 1, 2, 3, 5]]).all()


def test_empty_inputs():
    show("no rows")
    x = torch.empty((0, 40), device="cuda", requires_grad=True)
    w = torch.ones(40, device="cuda", requires_grad=True)
    b = torch.zeros(40, device="cuda", requires_grad=True)
    y = layers.layer_norm(x, w, b)
    gx, gw, gb = torch.autograd.grad(y, (x, w, b), torch.empty_like(y))
    assert gx.shape == (0, 40) and not gw.any() and not gb.any()
    y, s = layers.add_layer_norm(x, x.detach(), w, b, p=0.5, seed=1)
    assert y.shape == s.shape == (0, 40)
    assert layers.dropout(torch.empty((3, 0), device="cuda"), 0.5, 1).shape == (3, 0)
    wg = torch.randn((8, 40), device="cuda", requires_grad=True)
    wd = torch.randn((5, 8), device="cuda", requires_grad=True)
    y = layers.gated_ff(x, wg, wg.detach(), wd)
    assert y.shape == (0, 5)
    g = torch.autograd.grad(y, (x, wg, wd), torch.empty_like(y))
    assert g[0].shape == (0, 40) and not g[1].any() and not g[2].any()


# ---------------------------------------------------------------- orders and strides

def arranged(t, how):
    """The host tensor on the GPU, laid out in another way."""
    rows, width = t.shape
    if how == "slice":
        wide = torch.full((rows, width + 13), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 5:5 + width] = t.cuda()
        return wide[:, 5:5 + width]
    if how == "shifted":                                                     # an address that only the element type divides
        flat = torch.full((rows * width + 1,), float("nan"), dtype=t.dtype, device="cuda")
        flat[1:] = t.cuda().reshape(-1)
        return flat[1:].view(rows, width)
    if how == "transposed":
        return t.cuda().t().contiguous().t()
    if how == "every_second":
        wide = torch.full((2 * rows, width), float("nan"), dtype=t.dtype, device="cuda")
        wide[::2] = t.cuda()
        return wide[::2]
    if how == "columns_apart":
        wide = torch.full((rows, 2 * width), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, ::2] = t.cuda()
        return wide[:, ::2]
    return t.cuda()


ORDERS = ["slice", "shifted", "transposed", "every_second", "columns_apart"]


@pytest.mark.parametrize("how", ORDERS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width", [8, 37, 64, 520])
def test_orders(how, dtype, width):
    show("orders", how, dtype, width)
    x, r, dy, ds = (normal((21, width), dtype, 20 + i) for i in range(4))
    w, b = normal((width,), dtype, 24, 0.1, 1.0), normal((width,), dtype, 25)
    place = lambda t: arranged(t, how)  # noqa: E731
    check_norm(x, w, b, dy, place=place)
    check_add_norm(x, r, w, b, dy, ds, 0.3, place=place)
    results = []
    for put in (place, lambda t: t.cuda()):                                  # nothing is summed: the same bits
        leaf, add = put(x).requires_grad_(True), put(r).requires_grad_(True)
        y = layers.dropout(leaf, 0.3, 5, 6, residual=add)
        results.append([y, *torch.autograd.grad(y, [leaf, add], put(dy))])
    assert all(torch.equal(a, c) for a, c in zip(*results))


@pytest.mark.parametrize("how", ORDERS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,hidden,out", [(16, 32, 16), (33, 70, 9), (128, 64, 72)])
def test_orders_of_the_block(how, dtype, width, hidden, out):
    show("orders of the block", how, dtype, width, hidden, out)
    check_block(normal((50, width), dtype, 30), normal((hidden, width), dtype, 31, width ** -0.5), normal((hidden, width), dtype, 32, width ** -0.5),
                normal((out, hidden), dtype, 33, hidden ** -0.5), normal((50, out), dtype, 34), "silu", place=lambda t: arranged(t, how))


def test_broadcast_and_leading_axes():
    show("broadcast")
    row = normal((1, 40), torch.float32, 40).cuda().requires_grad_(True)
    x = row.expand(30, 40)
    y = layers.layer_norm(x)
    assert_within(y, host(layers.layer_norm(x.contiguous())), torch.full((), 16 * EPS32 * 8, dtype=torch.float64), "broadcast rows")
    g, = torch.autograd.grad(y, row, torch.ones((), device="cuda").expand(30, 40))
    assert g.shape == (1, 40)
    z = normal((3 * 5, 4 * 40), torch.float32, 41).cuda().view(3, 5, 160)[:, :, 40:80]
    y = layers.layer_norm(z)
    assert y.shape == (3, 5, 40) and torch.equal(y.reshape(15, 40), layers.layer_norm(z.reshape(15, 40)))
    cut = normal((6, 5 * 40), torch.float32, 42).cuda().view(6, 5, 40)[:, 1:4]                    # rows not at one distance
    assert torch.equal(layers.dropout(cut, 0.5, 3).reshape(18, 40), layers.dropout(cut.reshape(18, 40), 0.5, 3))
    v = normal((40,), torch.float32, 43).cuda()
    assert layers.layer_norm(v).shape == (40,)
    w = [normal((24, 40), torch.float32, 44).cuda(), normal((24, 40), torch.float32, 45).cuda(), normal((7, 24), torch.float32, 46).cuda()]
    assert torch.equal(layers.gated_ff(z, *w).reshape(15, 7), layers.gated_ff(z.reshape(15, 40), *w))
    assert layers.gated_ff(v, *w).shape == (7,)
    packed = torch.cat((w[0], w[1]))                                                              # gate and up as halves of one weight
    assert torch.equal(layers.gated_ff(v, packed[:24], packed[24:], w[2]), layers.gated_ff(v, *w))


# ---------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,p", [(1, 1, 0.5), (4096, 4, 0.5), (3, 8, 0.25), (7, 13, 0.1), (100, 64, 0.1), (5, 1001, 0.9), (2, 70000, 0.3),
                                          (9, 24, 0.0), (9, 24, 1.0), (300, 16, 1e-5)])
def test_dropout(rows, width, p, dtype):
    show("dropout", rows, width, p, dtype)
    seed, offset = 0xFEDCBA9876543210, (1 << 35) + 77
    x, r, dy = (normal((rows, width), dtype, 50 + i) for i in range(3))
    keep, scale = ref.keep_scale(rows, width, p, seed, offset)
    leaf, add = x.cuda().requires_grad_(True), r.cuda().requires_grad_(True)
    one = lambda t: torch.where(keep, t.float() * scale, torch.zeros(()))  # noqa: E731   (32 bits: one product, one sum, one rounding)
    y = layers.dropout(leaf, p, seed, offset)
    assert torch.equal(y.cpu(), one(x).to(dtype))
    assert torch.equal(torch.autograd.grad(y, leaf, dy.cuda())[0].cpu(), one(dy).to(dtype))
    y = layers.dropout(leaf, p, seed, offset, residual=add)
    want = torch.where(keep, x.double() * scale, torch.zeros((), dtype=torch.float64)) + r.double()
    assert_within(y, want, (UNIT[dtype] + EPS32) * want.abs() + 2 * EPS32 * (x.double().abs() * scale) + TINY[dtype], "y")
    gx, gr = torch.autograd.grad(y, (leaf, add), dy.cuda())
    assert torch.equal(gx.cpu(), one(dy).to(dtype)) and torch.equal(gr.cpu(), dy)


def test_dropped_elements_count_as_zero_whatever_they_hold():
    show("infinities under dropout")
    keep, scale = ref.keep_scale(40, 24, 0.5, 3, 4)
    x = torch.where(keep, torch.ones(()), torch.full((), float("nan")))
    x[0] = torch.where(keep[0], x[0], torch.full((), float("inf")))
    want = torch.where(keep, torch.full((), scale), torch.zeros(()))
    assert torch.equal(layers.dropout(x.cuda(), 0.5, 3, 4).cpu(), want)
    _, s = layers.add_layer_norm(x.cuda(), torch.zeros((40, 24), device="cuda"), p=0.5, seed=3, offset=4)
    assert torch.equal(s.cpu(), want)


def test_masks_of_different_seeds_and_offsets_have_nothing_in_common():
    show("independence of masks")
    x = torch.ones((1000, 1000), device="cuda")
    base = layers.dropout(x, 0.5, 1, 0) > 0
    assert abs(float(base.double().mean()) - 0.5) < 5 * 0.5e-3                                    # five deviations of a million draws
    for seed, offset in ((2, 0), (1, 1), (1 << 32 | 1, 0), (1, 1 << 32)):
        other = layers.dropout(x, 0.5, seed, offset) > 0
        assert abs(float((other == base).double().mean()) - 0.5) < 5 * 0.5e-3, (seed, offset)


def test_an_offset_in_gpu_memory_is_read_when_the_graph_runs():
    show("replayed graph")
    x, r = normal((50, 64), torch.float32, 60).cuda(), normal((50, 64), torch.float32, 61).cuda()
    w = [normal((96, 64), torch.float32, 62, 0.1).cuda(), normal((96, 64), torch.float32, 63, 0.1).cuda(), normal((64, 96), torch.float32, 64, 0.1).cuda()]
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    leaf = x.clone().requires_grad_(True)

    def step(at):
        y, s = layers.add_layer_norm(leaf, r, p=0.25, seed=9, offset=at)
        z = layers.dropout(layers.gated_ff(y, *w), 0.25, 10, at, residual=s)
        return z.detach(), *torch.autograd.grad(z, leaf, r)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(offset)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(offset)
    for number in (0, 1, 5, 1 << 33):
        offset.fill_(number)
        graph.replay()
        torch.cuda.synchronize()
        want = step(number)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), number
        torch.cuda.synchronize()


# ---------------------------------------------------------------- residual, dropout and norm in one

@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,p", [(1, 1, 0.0), (5, 24, 0.1), (40, 37, 0.25), (300, 32, 0.5), (70, 64, 0.1), (4, 1001, 0.25), (3, 1024, 0.1),
                                          (2, 8200, 0.3), (6, 40, 1.0), (33, 256, 0.0), (2, 20000, 0.1)])
def test_add_layer_norm(rows, width, p, dtype):
    show("add_layer_norm", rows, width, p, dtype)
    x, r = normal((rows, width), dtype, 70, 1.5, 0.3), normal((rows, width), dtype, 71, 2.0, -0.5)
    w, b = normal((width,), dtype, 72, 0.2, 1.0), normal((width,), dtype, 73)
    check_add_norm(x, r, w, b, normal((rows, width), dtype, 74), normal((rows, width), dtype, 75), p)


def check_add_norm(x, r, w, b, dy, ds, p, place=lambda t: t.cuda()):
    (rows, width), dtype = x.shape, x.dtype
    u, seed, offset = UNIT[dtype], 11, 1 << 40
    leaves = [*(place(t).requires_grad_(True) for t in (x, r)), *(t.cuda().requires_grad_(True) for t in (w, b))]
    y, s = layers.add_layer_norm(*leaves, p=p, seed=seed, offset=offset)
    X, R, W, B = (host(t) for t in (x, r, w, b))
    D = ref.dropped(X, p, seed, offset)
    S = D + R
    added = 2 * EPS32 * (D.abs() + R.abs())                                   # the sum before it is rounded
    assert_within(s, S, u * S.abs() + added + TINY[dtype], "s")
    rstd = 1 / torch.sqrt(S.var(1, unbiased=False, keepdim=True) + EPS)
    through = (added + added.mean(1, keepdim=True)) * rstd * (1 + norm(S, EPS).abs()) * W.abs()
    assert_within(y, ref.norm(S, W, B, EPS), norm_bound(S, W, B, u) + 2 * through + TINY[dtype], "y")
    dx, dr, dw, db = torch.autograd.grad([y, s], leaves, [place(dy), place(ds)])
    want, bound = check_norm_gradient(S, W, host(dy), dr, dw, db, u, UNIT[dtype], EPS, slack=u + 4 * EPS32, extra=host(ds))
    keep, scale = ref.keep_scale(rows, width, p, seed, offset)
    assert_within(dx, torch.where(keep, want * scale, torch.zeros((), dtype=torch.float64)),
                  torch.where(keep, (bound + (u + 2 * EPS32) * want.abs()) * scale, torch.zeros((), dtype=torch.float64)) + TINY[dtype], "dx")


def norm(S, eps):
    return ref.norm(S, None, None, eps)


def test_gradients_of_one_result_alone():
    show("one of two results")
    x, r = (normal((20, 48), torch.float32, 80 + i).cuda().requires_grad_(True) for i in range(2))
    w = normal((48,), torch.float32, 82, 0.1, 1.0).cuda().requires_grad_(True)
    g = normal((20, 48), torch.float32, 83).cuda()
    y, s = layers.add_layer_norm(x, r, w, p=0.4, seed=2)
    full = torch.autograd.grad([y, s], [x, r], [g, torch.zeros_like(g)], retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, [x, r], g, retain_graph=True), full))
    gx, gr = torch.autograd.grad(s, [x, r], g)
    assert torch.equal(gr, g) and torch.equal(gx, layers.dropout(g, 0.4, 2))
    y, s = layers.add_layer_norm(x, r, w, p=0.4, seed=2)
    (gw,) = torch.autograd.grad(y, [w], g)                                    # the parameters' alone
    y, s = layers.add_layer_norm(x, r, w, p=0.4, seed=2)
    assert torch.equal(gw, torch.autograd.grad(y, [x, r, w], g)[2])


# ---------------------------------------------------------------- gated feed-forward block

BLOCKS = [(1, 1, 1, 1), (1, 16, 32, 16), (2, 5, 3, 7), (3, 100, 33, 17), (17, 64, 64, 64), (16, 256, 512, 256), (31, 130, 66, 40), (33, 64, 128, 64),
          (64, 48, 200, 96), (65, 33, 129, 31), (100, 128, 96, 128), (128, 64, 256, 64), (200, 72, 136, 200), (257, 130, 258, 66), (300, 256, 300, 8),
          (1000, 64, 128, 64), (1025, 40, 72, 40), (4, 1000, 2731, 1000), (520, 96, 520, 520), (37, 512, 1025, 100), (1, 2048, 1024, 2048), (9, 24, 4096, 24),
          (300, 20, 200, 30), (500, 128, 128, 100), (77, 100, 64, 128), (4200, 32, 64, 32), (200, 64, 257, 64), (70, 129, 64, 32)]


@pytest.mark.parametrize("activation", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,hidden,out", BLOCKS)
def test_gated_ff(rows, width, hidden, out, dtype, activation):
    show("gated_ff", rows, width, hidden, out, dtype, activation)
    x = normal((rows, width), dtype, 90)
    wg, wu = normal((hidden, width), dtype, 91, width ** -0.5), normal((hidden, width), dtype, 92, width ** -0.5)
    wd, dy = normal((out, hidden), dtype, 93, hidden ** -0.5), normal((rows, out), dtype, 94)
    check_block(x, wg, wu, wd, dy, activation)


def check_block(x, wg, wu, wd, dy, activation, place=lambda t: t.cuda()):
    dtype = x.dtype
    (rows, width), hidden, out = x.shape, wg.shape[0], wd.shape[0]
    u, tiny = UNIT[dtype], TINY[dtype]
    leaves = [place(t).requires_grad_(True) for t in (x, wg, wu, wd)]
    y = layers.gated_ff(*leaves, activation=activation)
    X, WG, WU, WD, DY = (host(t) for t in (x, wg, wu, wd, dy))
    G, U = X @ WG.t(), X @ WU.t()
    A, SL = ref.act(activation, G), ref.slope(activation, G)
    H = A * U
    # products in 32 bits, then h rounded to the type; slopes of the activations are at most 1.13, their slopes at most 0.8
    eG, eU = (width + 4) * EPS32 * (X.abs() @ WG.abs().t()), (width + 4) * EPS32 * (X.abs() @ WU.abs().t())
    eA = 1.13 * eG + 8 * EPS32 * (A.abs() + G.abs())
    eH = eA * U.abs() + A.abs() * eU + eA * eU + (u + EPS32) * H.abs() + tiny
    Y = H @ WD.t()
    assert_within(y, Y, u * Y.abs() + (eH @ WD.abs().t()) + (hidden + 4) * EPS32 * (H.abs() @ WD.abs().t()) + tiny, "y")
    with torch.no_grad():
        plain = layers.gated_ff(*leaves, activation=activation)
    assert_within(plain, Y, u * Y.abs() + (eH @ WD.abs().t()) + (hidden + 4) * EPS32 * (H.abs() @ WD.abs().t()) + tiny, "y without a graph")

    dx, dwg, dwu, dwd = torch.autograd.grad(y, leaves, place(dy))
    DH = DY @ WD
    eDH = (out + 4) * EPS32 * (DY.abs() @ WD.abs())
    # g, u are saved in the type; act and its slope are taken at the saved g
    eg, eu = eG + u * G.abs() + tiny, eU + u * U.abs() + tiny
    bend = 0.0 if activation == "relu" else 0.8
    if activation == "relu":                                # a g within its error of 0 may go either way
        near = (G.abs() <= eg).double()
        eS = near
    else:
        eS = bend * eg + 16 * EPS32 * (1 + G.abs())
    DG, DU = DH * U * SL, DH * A
    both = lambda a, ea, b, eb: a.abs() * eb + ea * b.abs() + ea * eb  # noqa: E731
    eUS = both(U, eu, SL, eS)
    eDG = both(DH, eDH, U * SL, eUS) + (u + 4 * EPS32) * (DG.abs() + both(DH, eDH, U * SL, eUS)) + tiny
    eAs = 1.13 * eg + 8 * EPS32 * (A.abs() + G.abs())
    eDU = both(DH, eDH, A, eAs)
    eDU = eDU + (u + 4 * EPS32) * (DU.abs() + eDU) + tiny
    DX = DG @ WG + DU @ WU
    bound = eDG @ WG.abs() + eDU @ WU.abs() + (2 * hidden + 4) * EPS32 * (DG.abs() @ WG.abs() + DU.abs() @ WU.abs())
    assert_within(dx, DX, bound + u * DX.abs() + tiny, "dx")
    for got, d, e, other, name in ((dwg, DG, eDG, X, "dw_gate"), (dwu, DU, eDU, X, "dw_up")):
        want = d.t() @ other
        assert_within(got, want, e.t() @ other.abs() + (rows + 4) * EPS32 * (d.abs().t() @ other.abs()) + u * want.abs() + tiny, name)
    want = DY.t() @ H
    # h may be made again from the saved g and u
    eHs = both(A, eAs, U, eu) + (u + EPS32) * H.abs() + tiny
    assert_within(dwd, want, DY.abs().t() @ torch.maximum(eH, eHs) + (rows + 4) * EPS32 * (DY.abs().t() @ H.abs()) + u * want.abs() + tiny, "dw_down")


def test_block_gradients_that_are_not_asked_for():
    show("some gradients")
    t = [normal(s, torch.float32, 100 + i).cuda() for i, s in enumerate([(70, 32), (48, 32), (48, 32), (24, 48)])]
    dy = normal((70, 24), torch.float32, 104).cuda()
    leaves = [a.clone().requires_grad_(True) for a in t]
    full = torch.autograd.grad(layers.gated_ff(*leaves), leaves, dy)
    for i in range(4):
        leaves = [a.clone().requires_grad_(i == j) for j, a in enumerate(t)]
        assert torch.equal(torch.autograd.grad(layers.gated_ff(*leaves), leaves[i], dy)[0], full[i])


def test_large_and_infinite_gates():
    show("large gates")
    for activation in ("silu", "gelu", "relu"):
        x = torch.tensor([[300.0], [-300.0], [0.0], [30.0], [-30.0]], dtype=torch.float32)
        one = torch.ones((1, 1))
        y = layers.gated_ff(x.cuda(), one.cuda(), one.cuda(), one.cuda(), activation=activation)
        want = ref.act(activation, x.double()) * x.double()
        assert_within(y, want, 16 * EPS32 * want.abs() + 1e-30, activation)


# ---------------------------------------------------------------- differences

def by_differences(f, tensors, grads, results, step=2.0 ** -7):
    """Directional derivative of sum(result * grad) against the gradients, in 32 bits with the sums in 64."""
    torch.manual_seed(0)
    dirs = [torch.randn_like(t) for t in tensors]

    def value(sign):
        with torch.no_grad():
            out = f(*[t.detach() + sign * step * d for t, d in zip(tensors, dirs)])
        out = out if isinstance(out, tuple) else (out,)
        return sum(float((o.double() * g.double()).sum()) for o, g in zip(out, results))

    slope = (value(1.0) - value(-1.0)) / (2 * step)
    want = sum(float((g.double() * d.double()).sum()) for g, d in zip(grads, dirs))
    scale = sum(float((g.double() * d.double()).square().sum()) for g, d in zip(grads, dirs)) ** 0.5
    assert abs(slope - want) <= 1e-2 * max(abs(want), scale), (slope, want, scale)      # curvature: step^2, 6e-5, times third derivatives


@pytest.mark.parametrize("which", ["layer_norm", "add_layer_norm", "dropout", "silu", "gelu"])
def test_gradients_against_differences(which):
    show("differences", which)
    if which in ("silu", "gelu"):
        t = [normal((40, 24), torch.float32, 110), normal((56, 24), torch.float32, 111, 0.2), normal((56, 24), torch.float32, 112, 0.2),
             normal((20, 56), torch.float32, 113, 0.13)]
        f = lambda *a: layers.gated_ff(*a, activation=which)  # noqa: E731
    else:
        t = [normal((30, 40), torch.float32, 114), normal((30, 40), torch.float32, 115), normal((40,), torch.float32, 116, 0.1, 1.0),
             normal((40,), torch.float32, 117)]
        if which == "layer_norm":
            t, f = [t[0], t[2], t[3]], layers.layer_norm
        elif which == "add_layer_norm":
            f = lambda *a: layers.add_layer_norm(*a, p=0.25, seed=4, offset=2)  # noqa: E731
        else:
            t, f = t[:2], lambda a, r: layers.dropout(a, 0.25, 4, 2, residual=r)
    leaves = [a.cuda().requires_grad_(True) for a in t]
    out = f(*leaves)
    out = out if isinstance(out, tuple) else (out,)
    results = [torch.randn(o.shape, generator=gen(120)).cuda() for o in out]
    grads = torch.autograd.grad(out, leaves, results)
    by_differences(f, leaves, grads, results)


# ---------------------------------------------------------------- streams, repeats, other modes

def test_same_bits_every_time_and_on_other_streams():
    show("repeats")
    x, r = (normal((3000, 96), torch.bfloat16, 130 + i).cuda().requires_grad_(True) for i in range(2))
    w = normal((96,), torch.float32, 132).cuda().requires_grad_(True)
    b = normal((96,), torch.float32, 133).cuda().requires_grad_(True)
    ff = [normal(s, torch.bfloat16, 134, 0.1).cuda().requires_grad_(True) for s in ((160, 96), (160, 96), (96, 160))]
    g = normal((3000, 96), torch.bfloat16, 135).cuda()

    def step():
        y, s = layers.add_layer_norm(x, r, w, b, p=0.1, seed=1)
        z = layers.dropout(layers.gated_ff(y, *ff), 0.1, 2, residual=s)
        return [z, *torch.autograd.grad(z, [x, r, w, b, *ff], g)]

    first = step()
    for _ in range(3):
        assert all(torch.equal(a, c) for a, c in zip(first, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(first, other))


def test_inputs_changed_before_the_backward_pass_are_noticed():
    show("changed inputs")
    x = normal((8, 16), torch.float32, 140).cuda().requires_grad_(True)
    z = x * 1.0
    y = layers.layer_norm(z)
    z.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_more_than_reverse_mode_takes_autograds_own_function():
    show("other modes")
    x = normal((8, 16), torch.float32, 141).cuda()
    w = [normal(s, torch.float32, 142, 0.2).cuda() for s in ((24, 16), (24, 16), (16, 24))]
    other = normal((8, 16), torch.float32, 144).cuda()
    calls = [lambda t: layers.layer_norm(t), lambda t: layers.add_layer_norm(t, other, p=0.5, seed=1)[0], lambda t: layers.dropout(t, 0.5, 1),
             lambda t: layers.gated_ff(t, *w)]
    for f in calls:
        with torch.autograd.forward_ad.dual_level():
            with pytest.raises(Exception):
                f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        traced = torch.jit.trace(f, (x,), check_trace=False)
        assert torch.equal(traced(x * x + 1.0), f(x * x + 1.0))
    # the Functions themselves, as reverse mode would use them
    functions = layers._functions()
    leaf, r = x.clone().requires_grad_(True), (x * 0.5).requires_grad_(True)
    g = normal((8, 16), torch.float32, 143).cuda()
    for made, own in ((functions.norm.apply(leaf, r, None, None, 1e-5, 0.5, 1, 0), layers.add_layer_norm(leaf, r, p=0.5, seed=1)),
                      ((functions.dropout.apply(leaf, 0.5, 1, 0, r),), (layers.dropout(leaf, 0.5, 1, residual=r),))):
        assert all(torch.equal(a, b) for a, b in zip(made, own))
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(made[0], [leaf, r], g), torch.autograd.grad(own[0], [leaf, r], g)))
    leaves = [leaf, *(t.clone().requires_grad_(True) for t in w)]
    a, b = functions.gated.apply(*leaves, layers.SILU), layers.gated_ff(*leaves)
    assert torch.equal(a, b)
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(a, leaves, g), torch.autograd.grad(b, leaves, g)))


# ---------------------------------------------------------------- refusals

def test_refusals():
    show("refusals")
    x = torch.randn((6, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    wg, wd = torch.randn((24, 16), device="cuda"), torch.randn((16, 24), device="cuda")
    other = x.to(torch.bfloat16)
    calls = {
        "on the host": lambda: layers.layer_norm(x.cpu()),
        "of integers": lambda: layers.layer_norm(x.int()),
        "of doubles": lambda: layers.dropout(x.double(), 0.5, 1),
        "no tensor": lambda: layers.layer_norm([1.0, 2.0]),
        "no axis": lambda: layers.layer_norm(x[0, 0]),
        "empty rows": lambda: layers.layer_norm(x[:, :0]),
        "weight too short": lambda: layers.layer_norm(x, w[:15]),
        "weight of another type": lambda: layers.layer_norm(x, w.half()),
        "two parameter types": lambda: layers.layer_norm(other, w, w.to(torch.bfloat16)),
        "weight on the host": lambda: layers.layer_norm(x, w.cpu()),
        "negative eps": lambda: layers.layer_norm(x, w, eps=-1.0),
        "eps that is no number": lambda: layers.layer_norm(x, w, eps=float("nan")),
        "residual of another shape": lambda: layers.add_layer_norm(x, x[:5]),
        "residual of another type": lambda: layers.add_layer_norm(x, other),
        "broadcast residual": lambda: layers.dropout(x, 0.5, 1, residual=x[:1]),
        "rate above one": lambda: layers.dropout(x, 1.5, 1),
        "negative rate": lambda: layers.add_layer_norm(x, x, p=-0.1),
        "rate that is no number": lambda: layers.dropout(x, float("nan"), 1),
        "negative seed": lambda: layers.dropout(x, 0.5, -1),
        "seed beyond 64 bits": lambda: layers.dropout(x, 0.5, 1 << 64),
        "negative offset": lambda: layers.dropout(x, 0.5, 1, -1),
        "offset on the host": lambda: layers.dropout(x, 0.5, 1, torch.zeros(1, dtype=torch.int64)),
        "offset of 32 bits": lambda: layers.dropout(x, 0.5, 1, torch.zeros(1, dtype=torch.int32, device="cuda")),
        "two offsets": lambda: layers.dropout(x, 0.5, 1, torch.zeros(2, dtype=torch.int64, device="cuda")),
        "unknown activation": lambda: layers.gated_ff(x, wg, wg, wd, activation="tanh"),
        "gate of another width": lambda: layers.gated_ff(x, wg[:, :15], wg[:, :15], wd),
        "gate and up differ": lambda: layers.gated_ff(x, wg, wg[:23], wd),
        "down of another width": lambda: layers.gated_ff(x, wg, wg, wd[:, :23]),
        "weights of another type": lambda: layers.gated_ff(x, wg.half(), wg.half(), wd.half()),
        "weights of one axis": lambda: layers.gated_ff(x, wg[0], wg[0], wd),
        "empty hidden": lambda: layers.gated_ff(x, wg[:0], wg[:0], wd[:, :0]),
        "sparse": lambda: layers.layer_norm(x.to_sparse()),
    }
    for name, call in calls.items():
        with pytest.raises(dg.DgspError):
            call()
            pytest.fail(name)
    leaf = x.clone().requires_grad_(True)
    for y in (layers.layer_norm(leaf), layers.dropout(leaf, 0.5, 1), layers.gated_ff(leaf, wg, wg, wd)):
        with pytest.raises(RuntimeError, match="gradients of gradients"):
            torch.autograd.grad(y.sum(), leaf, create_graph=True)
    y = layers.layer_norm(leaf)
    y.sum().backward()
    with pytest.raises(RuntimeError):
        y.sum().backward()                                                    # the saved tensors are gone


def test_refusals_of_the_c_entry_points():
    """Nothing is enqueued: the status says what was wrong."""
    import ctypes
    show("refusals in C")
    L = layers.lib()
    x = torch.randn((6, 16), device="cuda")
    y = torch.empty_like(x)
    stream = torch.cuda.current_stream().cuda_stream
    good = layers.Dropout(0.5, 1, 0, None)
    P, bad = x.data_ptr(), dg.ERR_INVALID_ARG

    def drop(rows=6, width=16, type=0, d=good, xp=P, ldx=16, yp=y.data_ptr(), ldy=16):
        return L.dgsp_dropout(rows, width, type, ctypes.byref(d) if d is not None else None, xp, ldx, None, 0, yp, ldy, stream)

    assert drop() == dg.OK and drop(rows=0, xp=None, yp=None) == dg.OK
    assert drop(rows=-1) == bad and drop(type=3) == bad and drop(d=None) == bad and drop(xp=None) == bad and drop(yp=None) == bad
    assert drop(ldx=15) == bad and drop(ldy=15) == bad and drop(ldy=0) == bad and drop(d=layers.Dropout(1.01, 1, 0, None)) == bad
    assert drop(rows=(1 << 31)) == bad and drop(d=layers.Dropout(float("nan"), 1, 0, None)) == bad

    def norm(rows=6, width=16, type=0, ptype=0, residual=None, d=None, sum=None, ldx=16):
        return L.dgsp_layer_norm(rows, width, type, ptype, P, ldx, residual, 16, d, None, None, 1e-5, y.data_ptr(), 16, sum, 16, None, stream)

    assert norm() == dg.OK
    assert norm(width=0) == bad and norm(ptype=1) == bad and norm(type=1, ptype=2) == bad and norm(residual=P) == bad and norm(sum=P) == bad
    assert norm(d=ctypes.byref(good)) == bad and norm(ldx=3) == bad

    need = L.dgsp_gated_ff_workspace_bytes(6, 16, 24, 16, 0)
    w = torch.randn((24, 24), device="cuda")
    space = torch.empty(need + 16, dtype=torch.uint8, device="cuda")

    def gated(rows=6, width=16, hidden=24, out=16, type=0, act=0, ws=space.data_ptr(), size=need, ldg=24, saved=None):
        return L.dgsp_gated_ff(rows, width, hidden, out, type, act, P, 16, w.data_ptr(), ldg, w.data_ptr(), 24, w.data_ptr(), 24, y.data_ptr(), 16,
                               saved, ws, size, stream)

    assert gated() == dg.OK
    assert gated(width=0) == bad and gated(hidden=0) == bad and gated(act=3) == bad and gated(type=-1) == bad and gated(ldg=15) == bad
    assert gated(ws=None) == bad and gated(size=need - 1) == bad and gated(ws=space.data_ptr() + 4) == bad and gated(rows=-1) == bad
    assert gated(saved=space.data_ptr() + 4) == bad and gated(width=1 << 28) == bad
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows,width,p", [(60, 24, 0.0), (60, 24, 0.25), (9, 1001, 0.1), (3, 8200, 0.3)])
def test_gradient_of_the_weight_is_of_the_sum_before_it_is_rounded(rows, width, p, dtype):
    """With parameters in float nothing of 16 bits is left in it.  (s - mean) / spread is off by at most 2 (n + 8) e (|s| + mean |s|) /
    spread: s, the mean and the spread are sums of n terms at most; the sum over the rows adds (rows + 4) e of its magnitudes."""
    show("weight of add_layer_norm", rows, width, p, dtype)
    seed, offset = 11, 5
    x, r, dy, ds = (normal((rows, width), dtype, 120 + i, 1.0, 0.2) for i in range(4))
    w, b = normal((width,), torch.float32, 124, 0.1, 1.0), normal((width,), torch.float32, 125)
    on = [t.cuda().requires_grad_(True) for t in (x, r, w, b)]
    y, s = layers.add_layer_norm(*on, eps=EPS, p=p, seed=seed, offset=offset)
    torch.autograd.backward([y, s], [dy.cuda(), ds.cuda()])
    want = r.double() + ref.dropped(x.double(), p, seed, offset)
    _, dw, _ = ref.norm_gradient(want, w.double(), dy.double(), EPS)
    mean = want.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((want - mean) ** 2).mean(1, keepdim=True) + EPS)
    size = (dy.double().abs() * (want.abs() + want.abs().mean(1, keepdim=True)) * rstd).sum(0)
    assert_within(on[2].grad, dw, (2 * (width + 8) + rows + 4) * EPS32 * size, "dweight")
