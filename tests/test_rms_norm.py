"""Root-mean-square norm on the GPU against its definition in 64 bits.

Bounds, element by element.  With e = 2^-24: s is off by 2 e (|x| + |residual|) where it is a sum; the mean of n squares by (n + 4) e and what
the error of s makes of it, 1 / sqrt by half of that and 4 e; a product of three by 3 e; a result is rounded once, by u of itself."""
import pytest
import torch

import layer_reference as ref
import rows8_reference as ref8
from layer_reference import EPS32, TINY, UNIT, assert_within
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-5


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, dtype, seed, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float64) * scale + shift).to(dtype)


def host(t):
    return None if t is None else t.detach().double().cpu()


def definition(S, off, W, eps):
    """(y, bound of y before it is rounded, hat, bound of hat, rstd, its relative bound) of s, which the kernel has to `off`."""
    n = S.shape[1]
    rstd = 1 / torch.sqrt((S * S).mean(1, keepdim=True) + eps)
    relative = 0.5 * ((n + 4) * EPS32 + 2 * (S.abs() * off + off * off).mean(1, keepdim=True) * rstd ** 2) + 4 * EPS32
    hat = S * rstd
    hat_off = off * rstd + hat.abs() * (relative + EPS32)
    w = 1.0 if W is None else W
    return hat * w, (hat_off + 2 * EPS32 * hat.abs()) * abs(w), hat, hat_off, rstd, relative


def gradient(S, off, W, G, eps):
    """(ds, its bound, dweight, its bound), unrounded."""
    rows, n = S.shape
    _, _, hat, hat_off, rstd, relative = definition(S, off, W, eps)
    dhat = G if W is None else G * W
    q = (dhat * hat).mean(1, keepdim=True)
    q_off = ((n + 4) * EPS32 * (dhat * hat).abs() + dhat.abs() * hat_off).mean(1, keepdim=True)
    ds = (dhat - hat * q) * rstd
    size = dhat.abs() + hat.abs() * q.abs()
    ds_off = (4 * EPS32 * size + hat_off * q.abs() + (hat.abs() + hat_off) * q_off) * rstd + size * rstd * relative
    return ds, ds_off, (G * hat).sum(0), ((rows + 4) * EPS32 * (G * hat).abs() + G.abs() * hat_off).sum(0)


def check(x, r, w, dy, ds, p=0.0, eps=EPS, place=lambda t: t.cuda(), seed=3, offset=11):
    """Both passes of tensors on the host; without a residual r and ds are None."""
    u, up = UNIT[x.dtype], UNIT[(w if w is not None else x).dtype]
    leaves = [place(x).requires_grad_(True), None if r is None else place(r).requires_grad_(True), None if w is None else w.cuda().requires_grad_(True)]
    X, W, G = host(x), host(w), host(dy)
    if r is None:
        y, s = layers.rms_norm(leaves[0], leaves[2], eps), None
        S, off = X, torch.zeros_like(X)
    else:
        y, s = layers.add_rms_norm(leaves[0], leaves[1], leaves[2], eps, p, seed, offset)
        dropped = ref.dropped(X, p, seed, offset) if p else X
        S, off = host(r) + dropped, 2 * EPS32 * (host(r).abs() + dropped.abs())
        assert_within(s, S, u * S.abs() + off + TINY[x.dtype], "s")
    want, bound = definition(S, off, W, eps)[:2]
    assert_within(y, want, bound * (1 + u) + u * want.abs() + TINY[x.dtype], "y")
    with torch.no_grad():
        again = layers.rms_norm(leaves[0], leaves[2], eps) if r is None else layers.add_rms_norm(leaves[0], leaves[1], leaves[2], eps, p, seed, offset)[0]
        assert torch.equal(again, y)
    wanted = [t for t in leaves if t is not None]
    grads = torch.autograd.grad([y] if s is None else [y, s], wanted, [place(dy)] if s is None else [place(dy), place(ds)])
    if r is not None and x.dtype == torch.float32:                   # the backward pass reads the sum, as it was written
        S, off = host(s), torch.zeros_like(S)
    value, off, value_w, off_w = gradient(S, off, W, G, eps)
    if ds is not None:
        value, off = value + host(ds), off + 2 * EPS32 * (value.abs() + host(ds).abs())
    tiny = TINY[x.dtype]
    if r is None or not p:
        assert_within(grads[0], value, off * (1 + u) + u * value.abs() + tiny, "dx")
    else:
        keep, scale = ref.keep_scale(*x.shape, p, seed, offset)
        kept = keep * scale
        assert_within(grads[0], value * kept, (off * (1 + u) + u * value.abs() + 2 * EPS32 * value.abs()) * kept + tiny, "dx")
    if r is not None:
        assert_within(grads[1], value, off * (1 + u) + u * value.abs() + tiny, "dresidual")
    if w is not None:
        assert_within(grads[-1], value_w, off_w * (1 + up) + up * value_w.abs() + TINY[w.dtype], "dweight")
    return grads


SHAPES = [(1, 1), (1, 4096), (3, 2), (5, 3), (64, 7), (33, 8), (1025, 31), (257, 32), (63, 33), (7, 64), (9, 65), (65, 128), (6, 256), (5, 257), (3, 512),
          (3, 513), (5, 1001), (2, 2050), (3, 8192), (2, 8193), (1, 20000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", SHAPES)
def test_rms_norm(rows, width, dtype):
    print("[case] rms_norm", rows, width, dtype, flush=True)
    for params in {dtype, torch.float32}:
        check(normal((rows, width), dtype, 1, 2.0, 0.7), None, normal((width,), params, 2, 0.2, 1.0), normal((rows, width), dtype, 4), None)
    check(normal((rows, width), dtype, 5), None, None, normal((rows, width), dtype, 6), None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,p", [(1, 1, 0.0), (5, 24, 0.1), (40, 37, 0.25), (300, 32, 0.5), (4, 1001, 0.25), (3, 1024, 0.0), (2, 8200, 0.1), (9, 16, 1.0),
                                          (4100, 48, 0.0), (20000, 5, 0.1), (2600, 1000, 0.0)])
def test_add_rms_norm(rows, width, p, dtype):
    print("[case] add_rms_norm", rows, width, p, dtype, flush=True)
    x, r, dy, ds = (normal((rows, width), dtype, 10 + i) for i in range(4))
    check(x, r, normal((width,), torch.float32, 20, 0.2, 1.0), dy, ds, p)


def decoded(rows, shape):
    return ref8.read(rows.values, rows.scales, rows.width).view(shape)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", SHAPES + [(9, 96), (130, 40), (4099, 72), (2600, 520)])
def test_norms_in_8_bits(rows, width, dtype):
    """The scales are those of an amax within the bound of y, and each element is the nearest to a y within its bound: half a step, which is
    2^-4 of the element or 2^-10 of the scale."""
    print("[case] rms_norm_8bit", rows, width, dtype, flush=True)
    x, r = normal((rows, width), dtype, 30, 2.0), normal((rows, width), dtype, 31)
    w = normal((width,), torch.float32, 32, 0.2, 1.0)
    X, R, W = host(x), host(r), host(w)
    for add in (False, True):
        if add:
            y8, s = layers.add_rms_norm_8bit(x.cuda(), r.cuda(), w.cuda(), EPS)
            S, off = X + R, 2 * EPS32 * (X.abs() + R.abs())
            assert torch.equal(s, layers.add_rms_norm(x.cuda(), r.cuda(), w.cuda(), EPS)[1])
        else:
            y8, S, off = layers.rms_norm_8bit(x.cuda(), w.cuda(), EPS), X, torch.zeros_like(X)
        want, bound = definition(S, off, W, EPS)[:2]
        got = decoded(y8, want.shape)
        scale = 2.0 ** (y8.scales.cpu().transpose(0, 1).reshape(rows, -1)[:, :-(-width // 32)].double() - 127)
        amax, slack = ref8.cut(want).abs().amax(-1), ref8.cut(bound).amax(-1)
        assert bool(((amax - slack <= 448 * scale) & ((amax + slack >= 224 * scale) | (amax == 0))).all())
        per = scale.repeat_interleave(32, 1)[:, :width]
        assert_within(got, want, bound + torch.maximum(2.0 ** -4 * (want.abs() + bound), 2.0 ** -10 * per), "y in 8 bits")
        if not add:                                                  # of x itself all is made in 64 bits and rounded once
            values, exponents = ref8.quantised(want, "e4m3")
            assert torch.equal(y8.values.cpu().double().view(values.shape), values) and torch.equal(scale, 2.0 ** exponents.double())


@pytest.mark.gpu
def test_rows_that_leave_nothing():
    print("[case] zeros, infinities", flush=True)
    x = normal((6, 130), torch.float32, 40)
    x[1], x[2] = 0.0, 1e-20
    check(x, None, normal((130,), torch.float32, 41), normal((6, 130), torch.float32, 42), None)
    y = layers.rms_norm(torch.zeros((2, 40), device="cuda"), eps=0.0)
    assert torch.isnan(y).all()                                                            # 0 / 0, as the formula has it
    clean = layers.rms_norm(x.cuda())
    q = layers.rms_norm_8bit(x.cuda())
    for bad in (float("inf"), float("-inf"), float("nan")):
        z = x.clone()
        z[4, 77] = bad
        y = layers.rms_norm(z.cuda())
        other = [0, 1, 2, 3, 5]
        assert torch.equal(y[other], clean[other]) and torch.isnan(y[4, 77])
        q2 = layers.rms_norm_8bit(z.cuda())
        assert torch.equal(q2.values[other].view(torch.uint8), q.values[other].view(torch.uint8)) and torch.isnan(q2.values[4].float()[77])
    empty = torch.empty((0, 40), device="cuda", requires_grad=True)
    w = torch.ones(40, device="cuda", requires_grad=True)
    y = layers.rms_norm(empty, w)
    gx, gw = torch.autograd.grad(y, (empty, w), torch.empty_like(y))
    assert gx.shape == (0, 40) and not gw.any()
    with torch.no_grad():
        assert layers.rms_norm_8bit(empty).values.shape == (0, 64)


def arranged(t, how):
    rows, width = t.shape
    if how == "slice":
        wide = torch.full((rows, width + 13), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 5:5 + width] = t.cuda()
        return wide[:, 5:5 + width]
    if how == "shifted":
        flat = torch.full((rows * width + 1,), float("nan"), dtype=t.dtype, device="cuda")
        flat[1:] = t.cuda().reshape(-1)
        return flat[1:].view(rows, width)
    return t.cuda().t().contiguous().t()


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["slice", "shifted", "transposed"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_orders(how, dtype):
    print("[case] orders", how, dtype, flush=True)
    for width in (8, 37, 520):
        x, r, dy, ds = (normal((21, width), dtype, 50 + i) for i in range(4))
        w = normal((width,), dtype, 54, 0.1, 1.0)
        check(x, None, w, dy, None, place=lambda t: arranged(t, how))
        check(x, r, w, dy, ds, 0.3, place=lambda t: arranged(t, how))
        got, s = layers.add_rms_norm_8bit(arranged(x, how), arranged(r, how), w.cuda())
        want, plain = layers.add_rms_norm_8bit(x.cuda(), r.cuda(), w.cuda())
        assert torch.equal(got.values.view(torch.uint8), want.values.view(torch.uint8)) and torch.equal(got.scales, want.scales) and torch.equal(s, plain)


@pytest.mark.gpu
def test_broadcast_inputs_and_single_results():
    print("[case] broadcast", flush=True)
    row = normal((1, 40), torch.float32, 60).cuda().requires_grad_(True)
    x = row.expand(30, 40)
    y = layers.rms_norm(x)
    assert torch.equal(y, layers.rms_norm(x.contiguous()))
    g, = torch.autograd.grad(y, row, torch.ones((), device="cuda").expand(30, 40))
    assert g.shape == (1, 40)
    z = normal((15, 160), torch.float32, 61).cuda().view(3, 5, 160)[:, :, 40:80]
    assert torch.equal(layers.rms_norm(z).reshape(15, 40), layers.rms_norm(z.reshape(15, 40)))
    assert layers.rms_norm(z[0, 0]).shape == (40,)
    for dtype in TYPES:                                              # gradients of one result alone
        a, r = (normal((12, 40), dtype, 62 + i).cuda().requires_grad_(True) for i in range(2))
        w = normal((40,), dtype, 64).cuda().requires_grad_(True)
        gs = normal((12, 40), dtype, 65).cuda()
        y, s = layers.add_rms_norm(a, r, w)
        ga, gr, gw = torch.autograd.grad(s, (a, r, w), gs, allow_unused=True, retain_graph=True)
        assert torch.equal(ga, gs) and torch.equal(gr, gs) and gw is None
        zero = torch.autograd.grad((y, s), (a, r, w), (gs, torch.zeros_like(gs)), retain_graph=True)
        alone = torch.autograd.grad(y, (a, r, w), gs)
        assert all(torch.equal(p, q) for p, q in zip(zero, alone))


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["rms_norm", "add_rms_norm"])
def test_gradients_against_differences(which):
    """Central differences of steps h along random directions: off by h^2 / 6 times the third derivative, below 2^3 here, and by the
    rounding of the results, 2^-24 times the sum of their magnitudes, over h."""
    print("[case] differences", which, flush=True)
    t = [normal((30, 40), torch.float32, 70), normal((30, 40), torch.float32, 71), normal((40,), torch.float32, 72, 0.1, 1.0)]
    if which == "rms_norm":
        t, f = [t[0], t[2]], lambda *a: (layers.rms_norm(*a),)
    else:
        f = lambda *a: layers.add_rms_norm(*a, p=0.25, seed=4, offset=2)  # noqa: E731
    leaves = [a.cuda().requires_grad_(True) for a in t]
    out = f(*leaves)
    results = [torch.randn(o.shape, generator=gen(73)).cuda() for o in out]
    grads = torch.autograd.grad(out, leaves, results)
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        d = torch.randn(t[i].shape, generator=gen(74 + i)).cuda()
        with torch.no_grad():
            sides = [sum((o.double() * r.double()).sum() for o, r in zip(f(*(a + s * h * d if j == i else a for j, a in enumerate(leaves))), results)) for s in (1, -1)]
            size = sum((o.double() * r.double()).abs().sum() for o, r in zip(out, results))
        slope, want = (sides[0] - sides[1]) / (2 * h), (g.double() * d.double()).sum()
        bound = 8 * h * h / 6 * float((d.double().abs() ** 3).sum()) / d.numel() ** 0.5 + 2.0 ** -22 * float(size) / h
        assert abs(float(slope - want)) <= bound, (i, float(slope), float(want), bound)


@pytest.mark.gpu
def test_graph_capture_and_streams():
    print("[case] capture", flush=True)
    x, r = normal((50, 64), torch.bfloat16, 80).cuda(), normal((50, 64), torch.bfloat16, 81).cuda()
    w = normal((64,), torch.float32, 82, 0.1, 1.0).cuda().requires_grad_(True)
    leaf = x.clone().requires_grad_(True)
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(at):
        y, s = layers.add_rms_norm(leaf, r, w, p=0.25, seed=9, offset=at)
        with torch.no_grad():
            q, t = layers.add_rms_norm_8bit(leaf.detach(), r, w.detach())
        return [y.detach(), s.detach(), q.values.view(torch.uint8), q.scales, t, layers.dequantise(q), *torch.autograd.grad((y, s), (leaf, w), (r, r))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aside = step(offset)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(aside, step(0)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(offset)
    for number in (0, 1, 1 << 33):
        offset.fill_(number)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step(number))), number
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_other_modes_and_saved_tensors():
    print("[case] other modes", flush=True)
    x, other = normal((8, 16), torch.float32, 90).cuda(), normal((8, 16), torch.float32, 91).cuda()
    for f in (lambda t: layers.rms_norm(t), lambda t: layers.add_rms_norm(t, other, p=0.5, seed=1)[0]):
        with torch.autograd.forward_ad.dual_level(), pytest.raises(Exception):
            f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        traced = torch.jit.trace(f, (x,), check_trace=False)
        assert torch.equal(traced(x * x + 1.0), f(x * x + 1.0))
    with torch.autograd.forward_ad.dual_level(), pytest.raises(Exception):
        layers.rms_norm_8bit(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
    functions = layers._functions()
    for dtype in TYPES:
        leaves = [x.to(dtype).requires_grad_(True), other.to(dtype).requires_grad_(True), torch.ones(16, device="cuda", requires_grad=True)]
        g = normal((8, 16), dtype, 92).cuda()
        made, own = functions.rms.apply(*leaves, 1e-5, 0.5, 1, 0), layers.add_rms_norm(*leaves, p=0.5, seed=1)
        assert all(torch.equal(a, b) for a, b in zip(made, own))
        want = torch.autograd.grad(own, leaves, (g, g))
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(made, leaves, (g, g)), want))
        with torch.autograd.graph.save_on_cpu():
            out = layers.add_rms_norm(*leaves, p=0.5, seed=1)
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, (g, g)), want))
        shapes = {tuple(t.shape) for t in leaves}
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t if tuple(t.shape) in shapes else t[:-1]):
            out = layers.add_rms_norm(*leaves)
        with pytest.raises(RuntimeError, match="what the forward pass left"):
            torch.autograd.grad(out, leaves, (g, g))
        y = layers.rms_norm(leaves[0])
        with pytest.raises(RuntimeError, match="gradients of gradients"):
            torch.autograd.grad(y.sum(), leaves[0], create_graph=True)


@pytest.mark.gpu
def test_refusals():
    print("[case] refusals", flush=True)
    x, w = torch.randn((6, 16), device="cuda"), torch.ones(16, device="cuda")
    other = x.to(torch.bfloat16)
    calls = {
        "on the host": lambda f: f(x.cpu()),
        "of integers": lambda f: f(x.int()),
        "no tensor": lambda f: f([1.0]),
        "empty rows": lambda f: f(x[:, :0]),
        "weight too short": lambda f: f(x, w[:15]),
        "weight of another type": lambda f: f(x, w.half()),
        "weight on the host": lambda f: f(x, w.cpu()),
        "negative eps": lambda f: f(x, w, -1.0),
        "eps that is no number": lambda f: f(x, w, float("nan")),
    }
    for name, call in calls.items():
        for f in (layers.rms_norm, layers.rms_norm_8bit):
            with pytest.raises(dg.DgspError):
                call(f)
                pytest.fail(name)
    for f in (layers.add_rms_norm, layers.add_rms_norm_8bit):
        for residual in (x[:5], other, x.cpu(), None):
            with pytest.raises(dg.DgspError):
                f(x, residual)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(dg.DgspError):
            layers.add_rms_norm(x, x, p=p)
    for f in (lambda t: layers.rms_norm_8bit(t), lambda t: layers.add_rms_norm_8bit(x, t), lambda t: layers.rms_norm_8bit(x, t[0])):
        with pytest.raises(dg.DgspError, match="no gradient"):
            f(x.clone().requires_grad_(True))


@pytest.mark.gpu
def test_refusals_of_the_c_entry_points():
    import ctypes
    print("[case] refusals in C", flush=True)
    L, x = layers.lib(), torch.randn((6, 64), device="cuda")
    y, rstd, scales = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty((6, 4), dtype=torch.uint8, device="cuda")
    stream, bad, P, Y = torch.cuda.current_stream().cuda_stream, dg.ERR_INVALID_ARG, x.data_ptr(), y.data_ptr()
    drop = ctypes.byref(layers.Dropout(0.5, 1, 0, None))

    def norm(rows=6, width=64, type=0, ptype=0, residual=None, d=None, sum=None, ldx=64, yp=Y):
        return L.dgsp_rms_norm(rows, width, type, ptype, P, ldx, residual, 64, d, None, 1e-5, yp, 64, sum, 64, None, stream)

    assert norm() == dg.OK and norm(rows=0, yp=None) == dg.OK
    assert norm(width=0) == bad and norm(ptype=1) == bad and norm(residual=P) == bad and norm(sum=P) == bad and norm(d=drop) == bad
    assert norm(ldx=3) == bad and norm(yp=None) == bad and norm(rows=-1) == bad and norm(type=5) == bad and norm(rows=1 << 31) == bad

    def bits(rows=6, width=64, residual=None, sum=None, v=Y, ldv=64, s=scales.data_ptr(), ldx=64):
        return L.dgsp_rms_norm_8bit(rows, width, 0, 0, P, ldx, residual, 64, None, 1e-5, v, ldv, s, sum, 64, stream)

    assert bits() == dg.OK
    assert bits(width=0) == bad and bits(residual=P) == bad and bits(sum=P) == bad and bits(v=None) == bad and bits(v=Y + 4) == bad
    assert bits(ldv=48) == bad and bits(ldv=0) == bad and bits(s=None) == bad and bits(s=scales.data_ptr() + 1) == bad and bits(ldx=3) == bad

    need = L.dgsp_rms_norm_backward_workspace_bytes(6, 64)
    space, dw = torch.empty(need + 16, dtype=torch.uint8, device="cuda"), torch.empty(64, device="cuda")

    def back(rows=6, width=64, s=P, r=rstd.data_ptr(), dy=P, to=Y, d=None, dx=None, ws=space.data_ptr(), size=need):
        return L.dgsp_rms_norm_backward(rows, width, 0, 0, s, 64, None, 0, r, None, dy, 64, None, 0, d, to, dx, dw.data_ptr(), ws, size, stream)

    assert back() == dg.OK
    assert back(s=None) == bad and back(r=None) == bad and back(dy=None) == bad and back(to=None) == bad and back(d=drop) == bad and back(dx=P) == bad
    assert back(ws=None) == bad and back(size=need - 1) == bad and back(ws=space.data_ptr() + 4) == bad and back(width=0) == bad
    torch.cuda.synchronize()


def test_sizes_and_refusals_without_a_gpu():
    L, most = layers.lib(), (1 << 31) - 1 - 4096
    size = L.dgsp_rms_norm_backward_workspace_bytes
    assert size(0, 8) >= 0 and size(most, 64) > 0 and size(1, most) > 0
    for rows, width in ((-1, 8), (8, 0), (most + 1, 64), (1, most + 1), (1 << 62, 8), (8, (1 << 63) - 1)):
        assert size(rows, width) == 0
    x = torch.randn((4, 8))
    for call in (lambda: layers.rms_norm(x), lambda: layers.add_rms_norm(x, x), lambda: layers.rms_norm_8bit(x), lambda: layers.quantise(x)):
        with pytest.raises(dg.DgspError, match="GPU"):
            call()
    assert L.dgsp_rms_norm(4, 8, 0, 0, None, 8, None, 0, None, None, 1e-5, None, 8, None, 0, None, None) == dg.ERR_INVALID_ARG
    assert L.dgsp_quantise(4, 8, 0, 0, None, 8, None, 32, None, None) == dg.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(7, 24), (33, 64), (130, 513), (3, 1001), (300, 1001), (9, 2050), (3, 8192), (2, 8200), (2, 20000)])
def test_sums_in_8_bits_are_rounded_once(rows, width, dtype):
    """With a residual too every element is the nearest: s is the sum in 32 bits, and all that follows is made in 64."""
    print("[case] add_rms_norm_8bit", rows, width, dtype, flush=True)
    x, r, w = normal((rows, width), dtype, 95, 2.0), normal((rows, width), dtype, 96), normal((width,), torch.float32, 97, 0.2, 1.0)
    y8, s = layers.add_rms_norm_8bit(x.cuda(), r.cuda(), w.cuda(), EPS)
    S = x.float() + r.float()
    assert torch.equal(s.cpu(), S.to(dtype))
    values, exponents = ref8.quantised(definition(S.double(), torch.zeros_like(S, dtype=torch.float64), host(w), EPS)[0], "e4m3")
    scale = y8.scales.cpu().transpose(0, 1).reshape(rows, -1)[:, :exponents.shape[1]].long() - 127
    assert torch.equal(y8.values.cpu().double().view(values.shape), values) and torch.equal(scale, exponents.long())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("width", [3, 32, 300, 1001, 8200])
def test_rows_whose_squares_32_bits_cannot_hold(width, dtype, monkeypatch):
    """Large and small rows without eps: what counts is the sum of the squares, which passes 2^128 or ends below 2^-149.  Gradients of the largest row,
    some 1e-37 times differences of numbers near 1, may end below 2^-126, where steps stay as they are: 2^-149 in 32 bits, which the result is made in,
    and 2^-133 in bfloat16, half of which each rounding may take."""
    print("[case] range", width, dtype, flush=True)
    monkeypatch.setitem(TINY, dtype, 2.0 ** -150 + (2.0 ** -134 if dtype == torch.bfloat16 else 0.0))
    size = torch.tensor([1e25, 1e18, 1e37, 1.0, 1e-19, 1e-25, 1e-35], dtype=torch.float64)[:, None]
    x, r = ((normal((7, width), torch.float64, 90 + i) * size).to(dtype) for i in range(2))
    w, dy = normal((width,), dtype, 92, 0.2, 1.0), normal((7, width), dtype, 93)
    ds = (normal((7, width), torch.float64, 94) / size).to(dtype)
    check(x, None, w, dy, None, eps=0.0)
    check(x, r, w, dy, ds, eps=0.0)
    check(x, r, None, dy, ds, 0.25, eps=1e-30)
    with torch.no_grad():
        want = layers.rms_norm(x.cuda(), w.cuda(), 0.0)
        assert torch.isfinite(want).all() and (want != 0).any(1).all()
