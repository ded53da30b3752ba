"""The matrix product with its epilogue on the GPU against its definition in 64 bits (linear_reference.py has the bounds)."""
import pytest
import torch

import linear_reference as lin
import rows8_reference as ref8
from layer_reference import EPS32, assert_within
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

TYPES = [torch.float32, torch.bfloat16, torch.float16]
KINDS = [None, "silu", "gelu", "relu"]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float64) * scale).to(dtype)


def inputs(rows, width, out, dtype, params, seed=0):
    return [normal((rows, width), dtype, seed + 1), normal((out, width), dtype, seed + 2, width ** -0.5), normal((out,), params, seed + 3, 0.3),
            normal((rows, out), dtype, seed + 4), normal((rows, out), dtype, seed + 5)]


def double(t, device):
    return None if t is None else t.detach().to(device).double()


def check(t, kind, keep=False, place=lambda t: t.cuda(), at="cpu"):
    """Both passes; `t`: x, weight, bias, residual (both may be None) and dy on the host, `at`: where the definition is computed."""
    x, w, b, r, dy = t
    dtype, params = x.dtype, (b if b is not None else x).dtype
    leaves = [None if v is None else place(v).requires_grad_(True) for v in (x, w, b, r)]
    y = layers.linear(leaves[0], leaves[1], leaves[2], kind, leaves[3], keep_8bit=keep)
    X, W, B, R, G = (double(v, at) for v in t)
    (want, bound), (z, z_off) = lin.forward(X, W, B, kind, R, dtype)
    assert y.dtype == dtype
    assert_within(y, want.cpu(), bound.cpu(), "y")
    with torch.no_grad():
        assert torch.equal(layers.linear(leaves[0], leaves[1], leaves[2], kind, leaves[3]), y)
    kept = ref8.stands_for(x, "int8").to(at) if keep else X
    values = lin.backward(kept, W, z, z_off, kind, G, dtype, params, keep)
    there = [v for v in leaves if v is not None]
    grads = torch.autograd.grad(y, there, place(dy))
    for got, (value, bound), name in zip(grads, values, ("dx", "dweight", "dbias")[:3 if b is not None else 2]):
        assert_within(got, value.cpu(), bound.cpu(), name)
    if b is not None:
        assert grads[2].dtype == params
    if r is not None:
        assert torch.equal(grads[-1], place(dy))
    return y, grads


SIZES = [(1, 1, 1), (1, 4096, 200), (2, 3, 5), (5, 64, 64), (37, 100, 273), (129, 130, 131), (257, 33, 300), (300, 64, 32), (1000, 20, 64), (70, 1030, 515),
         (64, 8, 2048), (2050, 128, 16)]


FEW = [(16, 520, 70), (17, 300, 200), (32, 2049, 33), (33, 136, 1000), (64, 1000, 47), (65, 1000, 47)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", SIZES + FEW)
def test_linear(rows, width, out, dtype, kind):
    print("[case] linear", rows, width, out, dtype, kind, flush=True)
    for params in {dtype, torch.float32}:
        check(inputs(rows, width, out, dtype, params), kind)
    x, w, b, r, dy = inputs(rows, width, out, dtype, dtype, 7)
    check((x, w, None, None, dy), kind)
    check((x, w, b, None, dy), kind, keep=True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(1, 40, 24), (129, 130, 131), (300, 64, 64), (1000, 33, 40)])
def test_kept_in_8_bits(rows, width, out, dtype, kind):
    """The weight's gradient is that of x as it is kept, exactly so without an activation; the derivative's steps are the nearest."""
    print("[case] kept", rows, width, out, dtype, kind, flush=True)
    t = inputs(rows, width, out, dtype, torch.float32, 11)
    y, grads = check(t, kind, keep=True)
    whole = check(t, kind)
    assert torch.equal(y, whole[0])
    if kind in (None, "relu"):                                       # dx and dbias do not need what is rounded
        assert torch.equal(grads[0], whole[1][0]) and torch.equal(grads[2], whole[1][2])
    X, W, B, R, _ = (double(v, "cpu") for v in t)
    _, (z, z_off) = lin.forward(X, W, B, kind, R, dtype)
    saved = layers.native().linear_forward(*(v.cuda() for v in t[:3]), layers._epilogue(kind), t[3].cuda(), True)[1]
    if kind is None:
        assert saved.numel() == 0
        return
    codes = saved.view(torch.int8).cpu().view(rows, -1)[:, :out].double()
    off = (z.abs() <= z_off).double() if kind == "relu" else 0.8 * z_off + 8 * EPS32 * (1 + z.abs())
    assert_within(codes / 112, lin.slope(kind, z), 0.5 / 112 * (1 + 1e-9) + off, "steps")
    if kind == "relu":
        assert set(codes.unique().tolist()) <= {0.0, 112.0}


# rows, width, out: so that the tiles of 256, 128 and 64 are met, whole and at their ends, split along the depth and not
LARGE, MIDDLE, SPLIT = [(4096, 1024, 4096), (4099, 4088, 4100)], [(8192, 512, 512), (8185, 500, 522)], [(1, 4096, 16384), (130, 4099, 260), (16, 8192, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", LARGE + MIDDLE + SPLIT)
def test_tiles(rows, width, out, dtype):
    print("[case] tiles", rows, width, out, dtype, flush=True)
    check(inputs(rows, width, out, dtype, dtype, 21), "gelu", at="cuda")
    if rows != 4099:
        x, w, b, r, dy = inputs(rows, width, out, dtype, torch.float32, 22)
        check((x, w, b, None, dy), "silu", keep=True, at="cuda")


def arranged(t, how):
    if t.dim() == 1:
        wide = torch.full((2 * len(t),), float("nan"), dtype=t.dtype, device="cuda")
        wide[::2] = t.cuda()
        return wide[::2]
    rows, width = t.shape
    if how == "slice":
        wide = torch.full((rows, width + 13), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 5:5 + width] = t.cuda()
        return wide[:, 5:5 + width]
    if how == "shifted":
        flat = torch.full((rows * width + 1,), float("nan"), dtype=t.dtype, device="cuda")
        flat[1:] = t.cuda().reshape(-1)
        return flat[1:].view(rows, width)
    if how == "transposed":
        return t.cuda().t().contiguous().t()
    if how == "every_second":
        wide = torch.full((2 * rows, width), float("nan"), dtype=t.dtype, device="cuda")
        wide[::2] = t.cuda()
        return wide[::2]
    return torch._neg_view(-t.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["slice", "shifted", "transposed", "every_second", "negative"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,out", [(16, 16), (33, 70), (128, 72)])
def test_orders(how, dtype, width, out):
    print("[case] orders", how, dtype, width, out, flush=True)
    t = inputs(50, width, out, dtype, dtype, 31)
    for keep in (False, True):
        y, grads = check(t, "gelu", keep, place=lambda v: arranged(v, how))
        plain = check(t, "gelu", keep)
        assert torch.equal(y, plain[0]) and all(torch.equal(a, b) for a, b in zip(grads, plain[1]))


@pytest.mark.gpu
def test_leading_axes_broadcasts_and_empty_batches():
    print("[case] axes", flush=True)
    for dtype in TYPES:
        x, w, b, r, dy = (v.cuda() for v in inputs(30, 40, 24, dtype, dtype, 41))
        y = layers.linear(x, w, b, "silu", r)
        assert torch.equal(layers.linear(x.view(5, 6, 40), w, b, "silu", r.view(5, 6, 24)).view(30, 24), y)
        assert torch.equal(layers.linear(x[0], w, b, "silu", r[0]), layers.linear(x[:1], w, b, "silu", r[:1])[0])
        row, one = x[:1].clone().requires_grad_(True), r[:1].clone().requires_grad_(True)       # broadcast inputs
        for keep in (False, True):
            out = layers.linear(row.expand(30, 40), w, b, "silu", one.expand(30, 24), keep_8bit=keep)
            assert torch.equal(out, layers.linear(row.expand(30, 40).contiguous(), w, b, "silu", one.expand(30, 24).contiguous()))
            g = torch.autograd.grad(out, [row, one], dy)
            assert g[0].shape == (1, 40) and torch.equal(g[1], dy.sum(0, keepdim=True))
            wl = w.clone().requires_grad_(True)                                                  # a gradient that is one number
            out = layers.linear(x, wl, keep_8bit=keep)
            dw, = torch.autograd.grad(out.sum(), wl)
            same, = torch.autograd.grad(layers.linear(x, wl, keep_8bit=keep), wl, torch.ones_like(dy))
            assert torch.equal(dw, same)
        empty = torch.empty((0, 40), device="cuda", dtype=dtype, requires_grad=True)
        leaves = [empty, w.clone().requires_grad_(True), b.clone().requires_grad_(True)]
        for kind in KINDS:
            for keep in (False, True):
                out = layers.linear(*leaves, kind, keep_8bit=keep)
                assert out.shape == (0, 24)
                g = torch.autograd.grad(out, leaves, torch.empty_like(out))
                assert g[0].shape == (0, 40) and not g[1].any() and not g[2].any()
        tied = w.clone().requires_grad_(True)                                                    # the same tensor twice
        both, = torch.autograd.grad(layers.linear(tied, tied, None, "gelu"), tied, torch.ones((24, 24), device="cuda", dtype=dtype))
        a, c = tied.detach().clone().requires_grad_(True), tied.detach().clone().requires_grad_(True)
        parts = torch.autograd.grad(layers.linear(a, c, None, "gelu"), [a, c], torch.ones((24, 24), device="cuda", dtype=dtype))
        assert torch.equal(both, parts[0] + parts[1])


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
def test_gradients_that_are_not_asked_for(keep):
    print("[case] some gradients", keep, flush=True)
    for kind in (None, "gelu"):
        t = [v.cuda() for v in inputs(40, 72, 50, torch.bfloat16, torch.float32, 51)]
        full = [v.clone().requires_grad_(True) for v in t[:4]]
        want = torch.autograd.grad(layers.linear(full[0], full[1], full[2], kind, full[3], keep_8bit=keep), full, t[4])
        for mask in range(1, 16):
            leaves = [v.clone().requires_grad_(bool(mask >> i & 1)) for i, v in enumerate(t[:4])]
            asked = [i for i in range(4) if mask >> i & 1]
            y = layers.linear(leaves[0], leaves[1], leaves[2], kind, leaves[3], keep_8bit=keep)
            got = torch.autograd.grad(y, [leaves[i] for i in asked], t[4])
            assert all(torch.equal(g, want[i]) for g, i in zip(got, asked)), mask
        one, = torch.autograd.grad(layers.linear(full[0], full[1], full[2], kind, full[3], keep_8bit=keep), full[1:2], t[4])
        assert torch.equal(one, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_values_far_from_zero_and_not_finite(dtype):
    """z beyond the range of the type: the derivative is 0 or 1 there; an infinity or NaN stays in its row."""
    print("[case] far", dtype, flush=True)
    big = {torch.float32: 1e30, torch.bfloat16: 1e30, torch.float16: 6e4}[dtype]
    x = torch.tensor([[big, big], [-big, -big], [300.0, 300.0], [-300.0, -300.0]], dtype=dtype).cuda().requires_grad_(True)
    w = torch.ones((8, 2), device="cuda", dtype=dtype)
    for kind in ("silu", "gelu", "relu"):
        for keep in (False, True):
            y = layers.linear(x, w, None, kind, keep_8bit=keep)
            g, = torch.autograd.grad(y, x, torch.ones_like(y))
            assert torch.equal(g.float(), torch.tensor([8.0, 0.0, 8.0, 0.0], device="cuda")[:, None].expand(4, 2)), (kind, keep)
    t = [v.cuda() for v in inputs(70, 64, 72, dtype, dtype, 61)]
    clean = [t[0].clone().requires_grad_(True), t[1]]
    for bad in (float("inf"), float("nan")):
        dirty = t[0].clone()
        dirty[33, 5] = bad
        dirty.requires_grad_(True)
        for kind in KINDS:
            for keep in (False, True):
                pair = [layers.linear(v, t[1], None, kind, keep_8bit=keep) for v in (clean[0], dirty)]
                grads = [torch.autograd.grad(y, v, t[4])[0] for y, v in zip(pair, (clean[0], dirty))]
                rest = [i for i in range(70) if i != 33]
                assert torch.equal(pair[0][rest], pair[1][rest]) and torch.equal(grads[0][rest], grads[1][rest])
                if kind is None or bad != bad:
                    assert not torch.isfinite(pair[1][33]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu", None], ids=str)
def test_gradients_against_differences(kind):
    """As of the norm: h^2 / 6 times a third derivative below 2^3 per unit of the direction, and 2^-22 of the results' magnitudes over h."""
    print("[case] differences", kind, flush=True)
    t = [v.cuda() for v in inputs(40, 24, 56, torch.float32, torch.float32, 71)]
    leaves = [v.clone().requires_grad_(True) for v in t[:4]]
    f = lambda x, w, b, r: layers.linear(x, w, b, kind, r)  # noqa: E731
    grads = torch.autograd.grad(f(*leaves), leaves, t[4])
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        d = torch.randn(t[i].shape, generator=gen(72 + i)).cuda()
        d = d / d.norm()
        with torch.no_grad():
            sides = [(f(*(a + s * h * d if j == i else a for j, a in enumerate(leaves))).double() * t[4].double()).sum() for s in (1, -1)]
            size = float((f(*leaves).double() * t[4].double()).abs().sum())
        slope, want = float((sides[0] - sides[1]) / (2 * h)), float((g.double() * d.double()).sum())
        bound = 8 * h * h / 6 * float(t[4].abs().double().max()) * 3 ** 3 + 2.0 ** -22 * size / h
        assert abs(slope - want) <= bound, (i, slope, want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_capture_streams_and_repeats(dtype, keep):
    """The same bits every time, on another stream, and in every replay of a graph, also with new inputs; deep enough to be split."""
    print("[case] capture", dtype, keep, flush=True)
    for rows, width, out in ((30, 2050, 70), (300, 64, 64)):
        x, w, b, r, dy = (v.cuda() for v in inputs(rows, width, out, dtype, torch.float32, 81))
        leaves = [v.clone().requires_grad_(True) for v in (x, w, b)]

        def step():
            y = layers.linear(*leaves, "gelu", r, keep_8bit=keep)
            return [y.detach(), *torch.autograd.grad(y, leaves, dy)]

        want = step()
        assert all(torch.equal(a, c) for a, c in zip(step(), want))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            aside = step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(aside, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for turn in range(3):
            with torch.no_grad():
                leaves[0].mul_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(got, step())), turn
            torch.cuda.synchronize()


@pytest.mark.gpu
def test_other_modes_and_saved_tensors():
    print("[case] other modes", flush=True)
    for dtype in TYPES:
        for keep in (False, True):
            for kind in KINDS:
                t = [v.cuda() for v in inputs(30, 40, 24, dtype, torch.float32, 91)]
                leaves = [v.clone().requires_grad_(True) for v in t[:4]]
                call = lambda x, w, b, r: layers.linear(x, w, b, kind, r, keep_8bit=keep)  # noqa: E731
                y = call(*leaves)
                want = torch.autograd.grad(y, leaves, t[4])
                made = layers._functions().linear.apply(*leaves[:3], layers._epilogue(kind), leaves[3], keep)
                assert torch.equal(made, y) and all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(made, leaves, t[4]), want))
                with torch.autograd.graph.save_on_cpu():
                    out = call(*leaves)
                assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, t[4]), want))
                from torch.utils.checkpoint import checkpoint
                out = checkpoint(call, *leaves, use_reentrant=False)
                assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, t[4]), want))
                y = call(*leaves)
                with torch.no_grad():
                    leaves[1].add_(1.0)
                with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                    torch.autograd.grad(y, leaves, t[4])
                with pytest.raises(RuntimeError, match="gradients of gradients"):
                    torch.autograd.grad(call(*leaves).sum(), leaves[0], create_graph=True)
    x, w = torch.randn((8, 16), device="cuda"), torch.randn((4, 16), device="cuda")
    f = lambda t: layers.linear(t, w, None, "gelu")  # noqa: E731
    with torch.autograd.forward_ad.dual_level(), pytest.raises(Exception):
        f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
    assert torch.equal(torch.jit.trace(f, (x,), check_trace=False)(x + 1.0), f(x + 1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
def test_hooks_that_give_something_else_back_are_refused(keep):
    print("[case] hooks", keep, flush=True)
    t = [v.cuda() for v in inputs(30, 40, 24, torch.bfloat16, torch.bfloat16, 95)]
    for wrong in (lambda s: s[:-1], lambda s: s.cpu(), lambda s: s.to(torch.int16), lambda s: torch.cat((s, s))[::2].reshape(-1)):
        leaves = [v.clone().requires_grad_(True) for v in t[:2]]
        with torch.autograd.graph.saved_tensors_hooks(lambda s: s, wrong):
            y = layers.linear(*leaves, None, "gelu", keep_8bit=keep)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(y, leaves, t[4])


@pytest.mark.gpu
def test_what_is_kept_takes_an_eighth_or_a_quarter():
    """Of float and 16-bit matrices: x and the derivative take a byte an element and 1/32 for the scales."""
    print("[case] memory", flush=True)
    rows, width, out = 4096, 512, 256
    for dtype, whole in ((torch.float32, 4), (torch.bfloat16, 2)):
        w = torch.randn((out, width), device="cuda").to(dtype).requires_grad_(True)
        used = {}
        for keep in (False, True):
            x = torch.randn((rows, width), device="cuda").to(dtype).requires_grad_(True)
            before = torch.cuda.memory_allocated()
            y = layers.linear(x * 1.0, w, None, "gelu", keep_8bit=keep)
            used[keep] = torch.cuda.memory_allocated() - before - y.numel() * y.element_size()
            torch.autograd.grad(y.sum(), w)
            del x, y
        assert used[False] == rows * (width + out) * whole and used[True] == rows * (width + out) + rows * width // 32


@pytest.mark.gpu
def test_refusals():
    print("[case] refusals", flush=True)
    x, w = torch.randn((6, 16), device="cuda"), torch.randn((24, 16), device="cuda")
    b, r = torch.randn(24, device="cuda"), torch.randn((6, 24), device="cuda")
    f = layers.linear
    calls = {
        "unknown activation": lambda: f(x, w, b, "tanh"),
        "activation that is none": lambda: f(x, w, b, 3),
        "x on the host": lambda: f(x.cpu(), w),
        "weight on the host": lambda: f(x, w.cpu()),
        "of doubles": lambda: f(x.double(), w.double()),
        "two types": lambda: f(x, w.half()),
        "no tensor": lambda: f(x, None),
        "another width": lambda: f(x, w[:, :15]),
        "one axis": lambda: f(x, w[0]),
        "three axes": lambda: f(x, w[None]),
        "no columns": lambda: f(x, w[:0]),
        "no width": lambda: f(x[:, :0], w[:, :0]),
        "bias too short": lambda: f(x, w, b[:23]),
        "bias of two axes": lambda: f(x, w, b[None]),
        "bias of another type": lambda: f(x, w, b.half()),
        "bias on the host": lambda: f(x, w, b.cpu()),
        "broadcast residual": lambda: f(x, w, b, None, r[:1]),
        "residual of the input's shape": lambda: f(x, w, b, None, x),
        "residual of another type": lambda: f(x, w, b, None, r.half()),
        "residual on the host": lambda: f(x, w, b, None, r.cpu()),
        "sparse": lambda: f(x.to_sparse(), w),
    }
    for name, call in calls.items():
        with pytest.raises(dg.DgspError):
            call()
            pytest.fail(name)


@pytest.mark.gpu
def test_refusals_of_the_c_entry_points():
    print("[case] refusals in C", flush=True)
    L, bad = layers.lib(), dg.ERR_INVALID_ARG
    x, w, y = (torch.randn((24, 24), device="cuda") for _ in range(3))
    stream, X, W, Y = torch.cuda.current_stream().cuda_stream, x.data_ptr(), w.data_ptr(), y.data_ptr()
    need = max(L.dgsp_linear_workspace_bytes(6, 16, 24, 0), 16)
    space = torch.empty(4096 + need, dtype=torch.uint8, device="cuda")
    S = space.data_ptr()

    def there(rows=6, width=16, out=24, type=0, btype=0, act=0, keep=1, xp=X, ldx=16, ldw=16, r=None, yp=Y, ldy=24, saved=S, ws=S + 4096, size=need, v=None, ldv=32, s=S + 2048):
        return L.dgsp_linear(rows, width, out, type, btype, act, keep, xp, ldx, W, ldw, None, r, 24, yp, ldy, saved, v, ldv, s, ws, size, stream)

    assert there() == dg.OK and there(rows=0, xp=None, yp=None) == dg.OK and there(act=3, saved=None) == dg.OK and there(keep=0, saved=None) == dg.OK
    assert there(rows=-1) == bad and there(width=0) == bad and there(out=0) == bad and there(type=3) == bad and there(btype=1) == bad
    assert there(act=4) == bad and there(act=-1) == bad and there(keep=3) == bad and there(xp=None) == bad and there(ldx=15) == bad and there(ldw=15) == bad
    assert there(yp=None) == bad and there(ldy=23) == bad and there(ldy=0) == bad and there(saved=None) == bad and there(saved=S + 4) == bad
    assert there(width=1 << 22) == bad and there(rows=1 << 31) == bad
    assert there(keep=2, v=S + 1024) == dg.OK
    assert there(v=S + 1024) == bad and there(keep=2, v=S + 1028) == bad and there(keep=2, v=S + 1024, ldv=0) == bad and there(keep=2, v=S + 1024, s=None) == bad
    back_need = L.dgsp_linear_backward_workspace_bytes(6, 16, 24, 0, 0, 1)
    big = torch.empty(back_need + 16, dtype=torch.uint8, device="cuda")

    def back(rows=6, act=0, keep=1, xp=X, scales=None, wp=W, saved=S, dy=Y, dx=X, ws=big.data_ptr(), size=back_need, ldx=16):
        return L.dgsp_linear_backward(rows, 16, 24, 0, 0, act, keep, xp, ldx, scales, wp, 16, saved, dy, 24, dx, dx, None, ws, size, stream)

    out = torch.empty((64, 64), device="cuda")
    assert back(dx=out.data_ptr()) == dg.OK
    assert back(keep=0) == bad and back(xp=None) == bad and back(wp=None) == bad and back(saved=None) == bad and back(dy=None) == bad
    assert back(ws=None) == bad and back(size=back_need - 1) == bad and back(ws=big.data_ptr() + 4) == bad and back(act=9) == bad and back(ldx=3) == bad
    assert L.dgsp_linear_backward(6, 16, 24, 0, 0, 0, 2, X, 32, None, W, 16, S, Y, 24, out.data_ptr(), out.data_ptr(), None, big.data_ptr(), 1 << 40, stream) == bad
    torch.cuda.synchronize()


def test_sizes_without_a_gpu():
    L, most = layers.lib(), (1 << 31) - 1 - 4096
    for extents in ((-1, 8, 8), (most + 1, 8, 8), (8, 0, 8), (8, 8, 0), (8, 1 << 22, 8), (8, 8, 1 << 62)):
        assert L.dgsp_linear_workspace_bytes(*extents, 0) == 0 and L.dgsp_linear_backward_workspace_bytes(*extents, 0, 0, 1) == 0
    assert L.dgsp_linear_saved_bytes(-1, 8, 0, 0, 0, 1) == 0 and L.dgsp_linear_saved_bytes(8, 8, 0, 0, 0, 9) == 0 and L.dgsp_linear_saved_bytes(8, 8, 0, 0, 7, 1) == 0
    assert L.dgsp_linear_saved_bytes(8, 8, 0, 1, 0, 1) == 0
    for t, size in ((layers.F32, 4), (layers.BF16, 2), (layers.F16, 2)):
        for out, padded in ((1, 8), (8, 8), (33, 40)):
            assert L.dgsp_linear_saved_bytes(10, out, t, t, layers.GELU, 1) == 10 * padded * size and L.dgsp_linear_saved_bytes(10, out, t, t, layers.GELU, 2) == 10 * padded
            assert L.dgsp_linear_saved_bytes(10, out, t, layers.F32, layers.GELU, 1) == 10 * padded * 4
            assert L.dgsp_linear_saved_bytes(10, out, t, layers.F32, layers.RELU, 1) == 10 * padded and L.dgsp_linear_saved_bytes(10, out, t, t, layers.SILU, 0) == 0
            assert L.dgsp_linear_saved_bytes(10, out, t, t, layers.NO_ACTIVATION, 2) == 0
        for extents in ((0, 4096, 64), (0, 64, 4096), (0, 1, 1)):
            assert 0 <= L.dgsp_linear_workspace_bytes(*extents, t) <= L.dgsp_linear_workspace_bytes(1, *extents[1:], t)
            assert 0 <= L.dgsp_linear_backward_workspace_bytes(*extents, t, 0, 2) <= L.dgsp_linear_backward_workspace_bytes(1, *extents[1:], t, 0, 2)
    p = 1 << 20
    assert L.dgsp_linear(1 << 30, 8, 1 << 12, layers.F32, 0, 3, 0, p, 8, p, 8, None, None, 0, p, 1 << 12, None, None, 0, None, p, (1 << 63) - 1, None) == dg.ERR_UNSUPPORTED
    x = torch.randn((4, 8))
    with pytest.raises(dg.DgspError, match="GPU"):
        layers.linear(x, x)
    with pytest.raises(dg.DgspError, match="silu, gelu, relu"):
        layers.linear(x, x, activation="tanh")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS[1:])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(70, 64, 72), (70, 64, 64), (70, 200, 300), (9, 520, 40), (300, 2048, 260)])
def test_infinite_z_has_the_slope_of_a_number_far_from_zero(rows, width, out, dtype, kind):
    """1 or 0, whichever form is kept.  Of -1, 0 and 1, so that the columns that are not infinite have exact sums: the two forms keep the same x."""
    print("[case] infinite z", rows, width, out, dtype, kind, flush=True)
    x, w, dy = (torch.randint(-1, 2, shape, generator=gen(130 + i)).to(dtype).cuda() for i, shape in enumerate([(rows, width), (out, width), (rows, out)]))
    b = torch.zeros(out)
    b[1], b[5], b[out - 1], b[out - 2] = float("inf"), float("-inf"), float("inf"), float("-inf")
    found = []
    for params in (dtype, torch.float32):
        for keep in (False, True):
            leaves = [t.clone().requires_grad_(True) for t in (x, w, b.to(params).cuda())]
            y = layers.linear(*leaves, kind, keep_8bit=keep)
            found.append([g.detach() for g in torch.autograd.grad(y, leaves, dy)])
        saved = layers.native().linear_forward(x, w, b.to(params).cuda(), layers._epilogue(kind), None, True)[1]
        codes = saved.view(torch.int8).view(rows, -1)[:, :out]
        assert (codes[:, [1, out - 1]] == 112).all() and (codes[:, [5, out - 2]] == 0).all()
    for dx, dw, db in found:
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all() and torch.isfinite(db).all()
        for column, slope in ((1, 1), (5, 0), (out - 1, 1), (out - 2, 0)):
            assert torch.equal(dw[column], (slope * dy[:, column].double() @ x.double()).to(dtype))
            assert float(db[column]) == slope * float(dy[:, column].double().sum())


# rows, width, out: which of the two is faster by more than the clock's noise, bfloat16 (few_rows_kernels.hpp has the times)
FASTER_WITHOUT_TILES = [(1, 4096, 16384), (1, 4096, 1024), (16, 4096, 4096), (16, 2048, 256), (24, 2048, 4096), (24, 256, 20000), (32, 2048, 4096), (32, 1024, 16384),
                        (48, 1024, 8192), (64, 1024, 8192), (64, 1024, 1024), (1, 1024, 65536)]
FASTER_ON_TILES = [(1, 8192, 256), (1, 128, 65536), (16, 4096, 16384), (16, 512, 20000), (24, 4096, 512), (24, 256, 32768), (32, 2048, 256), (32, 2048, 512), (32, 2048, 1024),
                   (48, 512, 16384), (48, 256, 24576), (64, 512, 16384), (64, 512, 10240), (64, 2048, 512)]


@pytest.mark.parametrize("rows,width,out", FASTER_WITHOUT_TILES + FASTER_ON_TILES)
def test_few_rows_take_the_kernel_that_is_faster(rows, width, out):
    """Only tiles have a workspace."""
    assert (layers.lib().dgsp_linear_workspace_bytes(rows, width, out, layers.BF16) > 0) == ((rows, width, out) in FASTER_ON_TILES)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,out", [(1, 130, 40000), (16, 128, 20000), (20, 136, 24580), (24, 2040, 500), (30, 2048, 515), (40, 512, 10240), (64, 264, 16390)])
def test_few_rows_of_many_columns_and_deep_sums(rows, width, out):
    print("[case] few", rows, width, out, flush=True)
    check(inputs(rows, width, out, torch.bfloat16, torch.float32, 500), "gelu", at="cuda")
    x, w, b, r, dy = inputs(rows, width, out, torch.float16, torch.float16, 510)
    check((x, w, None, None, dy), None, keep=True, at="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("width,out", [(512, 256), (64, 64)])
def test_what_a_float_bias_keeps(width, out):
    """z in the bias's type, as its gradient is; kept in 8 bits, nothing more than with a bias of 16 bits."""
    print("[case] memory, float bias", width, out, flush=True)
    rows, dtype = 4096, torch.bfloat16
    w = torch.randn((out, width), device="cuda").to(dtype).requires_grad_(True)
    for params, of_z in ((dtype, 2), (torch.float32, 4)):
        b = torch.randn(out, device="cuda").to(params).requires_grad_(True)
        for keep in (False, True):
            x = torch.randn((rows, width), device="cuda").to(dtype).requires_grad_(True)
            before = torch.cuda.memory_allocated()
            y = layers.linear(x * 1.0, w, b, "gelu", keep_8bit=keep)
            used = torch.cuda.memory_allocated() - before - y.numel() * y.element_size()
            assert used == (rows * (width + out) + rows * 4 * -(-width // 128) if keep else rows * (2 * width + of_z * out)), (params, keep)
            assert torch.autograd.grad(y.sum(), b)[0].dtype == params
            del x, y
