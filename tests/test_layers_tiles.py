"""The gated feed-forward block on each of its matrix kernels against its definition in 64 bits, with bounds of what these kernels round.

The tiles are 64, 128 or 256 wide by the sizes of a product, and how operands lie in memory chooses between forms of them: the blocks here
run each form on each tile, with sums of several stages, at sizes that fill the tiles and at ones that do not.

Bounds, element by element, u = 2^-24, 2^-8, 2^-11 the half step of float32, bfloat16, float16 and e = 2^-24: a sum of n products in 32 bits is
off by (n + 4) e times the sum of the magnitudes.  act(g) adds 8 e (|act(g)| + |g|), its slope 16 e (1 + |g|).  h, dg and du are rounded
once, and so are results; act(g) and u act'(g), which the backward pass reads, are not.  Slopes of the activations are at most 1.13, theirs
at most 0.8 (relu: 1 where g is within its error of 0)."""
import re

import pytest
import torch

import layer_reference as ref
from layer_reference import EPS32, TINY, UNIT, assert_within
from paper_2106_16064_amd import layers

NAMES = ("y", "dx", "dw_gate", "dw_up", "dw_down")


def both(a, ea, b, eb):
    """The error of a product whose factors are off by ea and eb."""
    return a.abs() * eb + ea * b.abs() + ea * eb


def definition(x, wg, wu, wd, dy, activation, dtype):
    """Result and gradients in 64 bits, each with its bound; on the device of the operands."""
    u, e, tiny = UNIT[dtype], EPS32, TINY[dtype]
    (rows, width), hidden, out = x.shape, wg.shape[0], wd.shape[0]

    def rounded(v, off, once=u):
        return off + once * (v.abs() + off) + tiny

    g, up = x @ wg.t(), x @ wu.t()
    eg, eup = ((width + 4) * e * (x.abs() @ w.abs().t()) for w in (wg, wu))
    a, slope = ref.act(activation, g), ref.slope(activation, g)
    ea = 1.13 * eg + 8 * e * (a.abs() + g.abs())
    h = a * up
    eh = rounded(h, both(a, ea, up, eup), u + e)
    y = h @ wd.t()
    ey = rounded(y, eh @ wd.abs().t() + (hidden + 4) * e * ((h.abs() + eh) @ wd.abs().t()))

    dh, edh = dy @ wd, (out + 4) * e * (dy.abs() @ wd.abs())
    eslope = (g.abs() <= eg).double() if activation == "relu" else 0.8 * eg + 16 * e * (1 + g.abs())
    mul = up * slope
    emul = both(up, eup, slope, eslope) + 2 * e * mul.abs()
    dg, du = dh * mul, dh * a
    edg, edu = rounded(dg, both(dh, edh, mul, emul), u + 2 * e), rounded(du, both(dh, edh, a, ea), u + 2 * e)
    dx = dg @ wg + du @ wu
    edx = rounded(dx, edg @ wg.abs() + edu @ wu.abs() + (2 * hidden + 4) * e * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs()))
    found = [(y, ey), (dx, edx)]
    for d, ed in ((dg, edg), (du, edu)):
        w = d.t() @ x
        found.append((w, rounded(w, ed.t() @ x.abs() + (rows + 4) * e * ((d.abs() + ed).t() @ x.abs()))))
    w = dy.t() @ h
    found.append((w, rounded(w, dy.abs().t() @ eh + (rows + 4) * e * (dy.abs().t() @ (h.abs() + eh)))))
    return found


def operands(rows, width, hidden, out, dtype, device, seed=0):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen) * scale).to(dtype).to(device)

    return [normal(rows, width), normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5),
            normal(out, hidden, scale=hidden ** -0.5), normal(rows, out)]


def passes(t, activation):
    leaves = [v.detach().requires_grad_(True) for v in t[:4]]
    y = layers.gated_ff(*leaves, activation=activation)
    return [y.detach(), *torch.autograd.grad(y, leaves, t[4])]


def check(t, activation, dtype):
    want = definition(*(v.double() for v in t), activation, dtype)
    for got, (value, bound), name in zip(passes(t, activation), want, NAMES):
        assert_within(got, value.cpu(), bound.cpu(), name)
    with torch.no_grad():
        assert_within(layers.gated_ff(*t[:4], activation=activation), want[0][0].cpu(), want[0][1].cpu(), "y without a graph")


def tiles_of(call):
    """(edge, dual, A along k, B along k) of the matrix kernels that a call launches."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    names = [e.key for e in prof.key_averages()]
    found = set()
    for name in names:
        m = (re.search(r"tile_kernel<.*TileShape<(\d+), \d+, \d+, \d+, (true|false)>, (true|false), (true|false)", name)
             or re.search(r"tile_kernelI\w*?9TileShapeILi(\d+)ELi\d+ELi\d+ELi\d+ELb([01])EEELb([01])ELb([01])E", name))     # not every name is demangled
        if m:
            found.add((int(m[1]), *(v in ("true", "1") for v in m.groups()[1:])))
    assert found, names
    return found


UP, DOWN, BACK, WEIGHTS = (True, True, True), (False, True, True), (False, True, False), (False, False, False)
FORMS = {UP, DOWN, BACK, WEIGHTS}

# rows, width, hidden, out: the tiles' edge in all four forms
LARGE = [(4096, 4096, 4096, 4096), (4099, 4088, 4100, 4090)]
MIDDLE = [(8192, 512, 512, 512), (4096, 256, 1024, 256), (8185, 500, 522, 499)]
SMALL = [(100, 256, 300, 130), (130, 512, 200, 72), (97, 250, 333, 131)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("edge,block", [(edge, block) for edge, blocks in ((256, LARGE), (128, MIDDLE), (64, SMALL)) for block in blocks], ids=str)
def test_tiles_of_16_bit_types(edge, block, dtype):
    print("[case] tiles", edge, block, dtype, flush=True)
    activation = "silu" if dtype == torch.bfloat16 else "gelu"
    t = operands(*block, dtype, "cuda")
    assert tiles_of(lambda: passes(t, activation)) == {(edge, *form) for form in FORMS}
    check(t, activation, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("edge,block", [(128, (4096, 256, 1024, 256)), (128, (8192, 512, 512, 512)), (128, (4099, 250, 1030, 513)), (64, (100, 256, 300, 130)),
                                        (64, (97, 250, 333, 131))], ids=str)
def test_tiles_of_float(edge, block):
    print("[case] tiles", edge, block, "float", flush=True)
    t = operands(*block, torch.float32, "cuda")
    assert tiles_of(lambda: passes(t, "gelu")) == {(edge, *form) for form in FORMS}
    check(t, "gelu", torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("edge,block", [(256, (4099, 4088, 4100, 4090)), (128, (8185, 500, 522, 499)), (64, (97, 250, 333, 131))], ids=str)
def test_tiles_of_views(edge, block):
    """Rows that are column slices of wider ones: read in place where they begin and end on 16 bytes."""
    print("[case] tiles of views", edge, block, flush=True)
    for first in (8, 3):
        wide = [torch.full((v.shape[0], v.shape[1] + 24), float("nan"), dtype=v.dtype, device="cuda") for v in operands(*block, torch.bfloat16, "cuda")]
        t = []
        for w, v in zip(wide, operands(*block, torch.bfloat16, "cuda", seed=1)):
            w[:, first:first + v.shape[1]] = v
            t.append(w[:, first:first + v.shape[1]])
        assert edge in {found[0] for found in tiles_of(lambda: passes(t, "relu"))}
        check(t, "relu", torch.bfloat16)


# One row, so that each gradient of a weight is a single product and its error that of the factors: rounding more than is said shows.
SINGLE = [(1, 8, 300, 8), (1, 24, 1000, 5), (1, 33, 700, 17), (1, 8, 64, 8), (1, 40, 200, 40), (1, 100, 128, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("block", SINGLE, ids=str)
def test_what_is_rounded_of_single_products(block, dtype, activation):
    print("[case] single products", block, dtype, activation, flush=True)
    for seed in range(4):
        check(operands(*block, dtype, "cuda", seed=seed), activation, dtype)


def beyond(got, want):
    return [name for (value, bound), v, name in zip(want, got, NAMES) if ((v - value).abs() > bound).any()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("block", SINGLE[:3], ids=str)
def test_the_bounds_tell_what_is_rounded(block, dtype):
    """A model of the block on the host: with the roundings that are said it is within the bounds, with act(g) and u act'(g) in 16 bits, or
    with g and u in 16 bits, the gradients of the gates' weights are not."""
    def model(t, of_factors, of_gates):
        x, wg, wu, wd, dy = (v.double() for v in t)
        once = lambda v: v.to(dtype).double()  # noqa: E731
        g, up = x @ wg.t(), x @ wu.t()
        h = once(ref.act("silu", g) * up)
        if of_gates:
            g, up = once(g), once(up)
        a, mul = ref.act("silu", g), up * ref.slope("silu", g)
        if of_factors:
            a, mul = once(a), once(mul)
        dh = dy @ wd
        dg, du = once(dh * mul), once(dh * a)
        return [once(v) for v in (h @ wd.t(), dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h)]

    wrong = {True: set(), False: set()}
    for seed in range(4):
        t = operands(*block, dtype, "cpu", seed=seed)
        want = definition(*(v.double() for v in t), "silu", dtype)
        assert beyond(model(t, False, False), want) == []
        for of_factors in (True, False):
            wrong[of_factors] |= set(beyond(model(t, of_factors, not of_factors), want))
    assert {"dw_gate", "dw_up"} <= wrong[True] and {"dw_gate", "dw_up"} <= wrong[False]


# width, hidden, out of every padded shape of the kernels that hold the weights, filling it and not
NARROW = [(32, 64, 32), (30, 50, 7), (32, 128, 32), (20, 100, 31), (32, 256, 32), (9, 200, 24), (64, 64, 64), (33, 64, 40), (64, 128, 64), (60, 72, 50),
          (64, 256, 64), (40, 130, 64), (128, 64, 128), (72, 33, 100), (128, 128, 128), (127, 128, 65)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("block", NARROW, ids=str)
def test_narrow_blocks_of_many_rows(block, dtype):
    """So many that workgroups go on to a second and a third tile, the last of which is not full."""
    print("[case] narrow", block, dtype, flush=True)
    t = operands(2 * 256 * 128 + 2 * 128 + 37, *block, dtype, "cuda")
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        passes(t, "silu")
        torch.cuda.synchronize()
    names = " ".join(e.key for e in prof.key_averages())
    assert "narrow_forward_kernel" in names and "narrow_backward" in names and "tile_kernel" not in names
    check(t, "silu", dtype)
