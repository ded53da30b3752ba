"""The product of rows in 8 bits on the GPU: its operands' values are known exactly, so that what is left are the sums, the epilogue and one
rounding (linear_reference.py has the bounds, and what the matrix instruction cuts off of sums of eight)."""
import pytest
import torch

import linear_reference as lin
import rows8_reference as ref8
from layer_reference import EPS32, assert_within
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def spread(rows, width, seed, scale=1.0):
    """Blocks whose scales differ by up to 2^8."""
    x = torch.randn((rows, width), generator=gen(seed)) * scale
    return x * 2.0 ** torch.randint(-4, 5, (rows, -(-width // 32)), generator=gen(seed + 1)).float().repeat_interleave(32, 1)[:, :width]


def scales_of(t):
    rows = t.scales.shape[1]
    return 2.0 ** (t.scales.cpu().transpose(0, 1).reshape(rows, -1)[:, :-(-t.width // 32)].double() - 127)


def check(rows, width, out, dtype, kind, seed=0, residual=True, at="cpu"):
    x8, w8 = layers.quantise(spread(rows, width, seed).cuda()), layers.quantise(spread(out, width, seed + 2, width ** -0.5).cuda())
    b = torch.randn(out, generator=gen(seed + 4))
    r = torch.randn((rows, out), generator=gen(seed + 5)).to(dtype) if residual else None
    y = layers.linear_8bit(x8, w8, b.cuda(), kind, None if r is None else r.cuda(), dtype)
    X, W = (ref8.read(*t).to(at) for t in (x8, w8))
    lost = lin.cut_off_in_8bit(X, W, scales_of(x8).to(at), scales_of(w8).to(at))
    (want, bound), _ = lin.forward(X, W, b.double().to(at), kind, None if r is None else r.double().to(at), dtype, lost)
    assert y.dtype == dtype
    assert_within(y, want.cpu(), bound.cpu(), "y")
    return x8, w8, b, y


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [None, "silu", "gelu", "relu"], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(1, 1, 1), (1, 4096, 200), (2, 3, 5), (5, 31, 64), (16, 32, 16), (37, 100, 273), (129, 130, 131), (64, 128, 64), (65, 160, 63),
                                            (257, 33, 300), (70, 1030, 515), (3, 257, 2048), (17, 300, 200), (32, 2049, 33), (33, 136, 1000), (64, 1500, 47), (65, 1500, 47)])
def test_linear_8bit(rows, width, out, dtype, kind):
    print("[case] linear_8bit", rows, width, out, dtype, kind, flush=True)
    check(rows, width, out, dtype, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(4096, 2048, 4096), (4099, 2100, 4100), (8192, 512, 512), (8185, 500, 522), (1, 4096, 16384), (130, 4099, 260), (16, 8192, 64)])
def test_tiles(rows, width, out, dtype):
    print("[case] tiles", rows, width, out, dtype, flush=True)
    check(rows, width, out, dtype, "gelu", 11, at="cuda")
    check(rows, width, out, dtype, None, 12, residual=False, at="cuda")


@pytest.mark.gpu
def test_each_block_has_its_own_scale():
    """Operands of ones, so that the product is a sum of products of scales: which scale goes with which 32 columns."""
    print("[case] scales", flush=True)
    for rows, out, blocks in ((64, 64, 4), (64, 64, 9), (300, 300, 16), (8192, 512, 17)):
        width = 32 * blocks
        e = torch.randint(-6, 7, (rows, blocks), generator=gen(1))
        f = torch.randint(-6, 7, (out, blocks), generator=gen(2))
        ones = lambda n: torch.ones((n, width)).to(torch.float8_e4m3fn).cuda()  # noqa: E731

        def laid(t):
            whole = torch.full((t.shape[0], -(-blocks // 4) * 4), 127, dtype=torch.uint8)
            whole[:, :blocks] = (t + 127).to(torch.uint8)
            return whole.view(t.shape[0], -1, 4).transpose(0, 1).contiguous().cuda()

        y = layers.linear_8bit(layers.Rows8(ones(rows), laid(e), width), layers.Rows8(ones(out), laid(f), width), dtype=torch.float32)
        want = 32 * (2.0 ** e.double()) @ (2.0 ** f.double()).t()
        # the products of a block are equal and lose nothing, but the sums span 2^-7 ... 2^21, more than 24 bits: each of their additions, all
        # of positive numbers, is off by at most 2^-24 of a number that is at most the result
        assert_within(y, want, (width + 4) * EPS32 * want, "y")


@pytest.mark.gpu
def test_orders_axes_and_edges():
    print("[case] orders", flush=True)
    x8, w8, b, y = check(24, 200, 40, torch.bfloat16, "silu", 21, residual=False)
    f = lambda x, w: layers.linear_8bit(x, w, b.cuda(), "silu")  # noqa: E731
    Rows8 = layers.Rows8

    def apart(t, first, step):
        wide = torch.full((t.values.shape[0], t.values.shape[1] + step), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        wide.view(torch.uint8)[:, first:first + t.values.shape[1]] = t.values.view(torch.uint8)
        return Rows8(wide[:, first:first + t.values.shape[1]], t.scales, t.width)

    for first, step in ((0, 32), (16, 64), (3, 40)):
        assert torch.equal(f(apart(x8, first, step), w8), y) and torch.equal(f(x8, apart(w8, first, step)), y)
    for t in (x8, w8):
        other = Rows8(t.values.t().contiguous().t(), t.scales.transpose(0, 1).contiguous().transpose(0, 1), t.width)
        assert torch.equal(f(other, w8) if t is x8 else f(x8, other), y)
    axes = f(Rows8(x8.values.view(2, 12, 224), x8.scales, 200), w8)
    assert axes.shape == (2, 12, 40) and torch.equal(axes.view(24, 40), y)
    one = f(Rows8(x8.values[3], x8.scales[:, 3:4], 200), w8)
    assert one.shape == (40,) and torch.equal(one, f(Rows8(x8.values[3:4], x8.scales[:, 3:4], 200), w8)[0])
    same = f(Rows8(x8.values[:1].expand(24, 224), x8.scales[:, :1].expand(2, 24, 4), 200), w8)
    assert torch.equal(same, f(Rows8(x8.values[:1].repeat(24, 1), x8.scales[:, :1].repeat(1, 24, 1), 200), w8))
    assert f(layers.quantise(torch.empty((0, 200), device="cuda")), w8).shape == (0, 40)
    for bad in (float("inf"), float("nan")):                         # stays in its row
        x = spread(24, 200, 21)
        x[7, 150] = bad
        got = f(layers.quantise(x.cuda()), w8)
        rest = [i for i in range(24) if i != 7]
        assert torch.equal(got[rest], y[rest]) and torch.isnan(got[7]).all()


@pytest.mark.gpu
def test_a_run_of_the_serving_form():
    """Norm, product, norm, product as a program would chain them, captured and replayed with new inputs; and next to the whole ones: the
    two quantised operands of a product are each within 2^-4 of themselves, so the product is within (2^-3 + 2^-8) sum |x| |w|."""
    print("[case] serving", flush=True)
    torch.manual_seed(0)
    x, r = torch.randn((33, 96), device="cuda", dtype=torch.bfloat16), torch.randn((33, 96), device="cuda", dtype=torch.bfloat16)
    g = torch.ones(96, device="cuda")
    up, down = torch.randn((200, 96), device="cuda") * 0.1, torch.randn((96, 200), device="cuda") * 0.1
    up8, down8 = layers.quantise(up), layers.quantise(down)

    def block():
        h, s = layers.add_rms_norm_8bit(x, r, g)
        u = layers.linear_8bit(h, up8, None, "gelu")
        return layers.linear_8bit(layers.quantise(u), down8, None, None, s), u, h, s

    y, u, h, s = block()
    whole = layers.rms_norm(s.float(), g)
    z = layers.linear(whole, up)
    size = whole.abs().double() @ up.abs().double().t()
    small = (2.0 ** -9 * 32 ** 0.5) * size.max()                      # elements below 2^-6 of their scale are rounded to steps of 2^-9 of it
    first = layers.linear_8bit(h, up8, dtype=torch.float32)
    assert bool(((first - z).abs().double() <= (2.0 ** -3 + 2.0 ** -7) * size + small).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aside = block()[0]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(aside, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block()[0]
    for _ in range(3):
        x.mul_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, block()[0])
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_refusals():
    print("[case] refusals", flush=True)
    x, w = torch.randn((6, 100), device="cuda"), torch.randn((24, 100), device="cuda")
    x8, w8, Rows8, f = layers.quantise(x), layers.quantise(w), layers.Rows8, layers.linear_8bit
    b = torch.randn(24, device="cuda")
    calls = {
        "whole numbers": lambda: f(layers.quantise(x, "int8"), w8),
        "whole weights": lambda: f(x8, layers.quantise(w, "int8")),
        "no rows in 8 bits": lambda: f(x, w),
        "unknown activation": lambda: f(x8, w8, None, "tanh"),
        "another width": lambda: f(x8, layers.quantise(w[:, :99])),
        "weight of three axes": lambda: f(x8, Rows8(w8.values[None], w8.scales, 100)),
        "no columns": lambda: f(x8, layers.quantise(w[:0])),
        "scales of fewer rows": lambda: f(x8, Rows8(w8.values, w8.scales[:, :23], 100)),
        "scales of a group less": lambda: f(layers.quantise(torch.randn((6, 200), device="cuda")), Rows8(layers.quantise(torch.randn((24, 200), device="cuda")).values, w8.scales, 200)),
        "weight on the host": lambda: f(x8, Rows8(w8.values.cpu(), w8.scales.cpu(), 100)),
        "bias too short": lambda: f(x8, w8, b[:23]),
        "bias of another type": lambda: f(x8, w8, b.half()),
        "bias with a gradient": lambda: f(x8, w8, b.clone().requires_grad_(True)),
        "residual of another type": lambda: f(x8, w8, b, None, torch.randn((6, 24), device="cuda")),
        "residual of another shape": lambda: f(x8, w8, b, None, torch.randn((5, 24), device="cuda").bfloat16()),
        "of doubles": lambda: f(x8, w8, dtype=torch.float64),
    }
    for name, call in calls.items():
        with pytest.raises(dg.DgspError):
            call()
            pytest.fail(name)


@pytest.mark.gpu
def test_refusals_of_the_c_entry_point():
    print("[case] refusals in C", flush=True)
    L, bad = layers.lib(), dg.ERR_INVALID_ARG
    x8, w8 = layers.quantise(torch.randn((6, 100), device="cuda")), layers.quantise(torch.randn((24, 100), device="cuda"))
    y = torch.empty((6, 24), device="cuda")
    stream, X, W, XS, WS = torch.cuda.current_stream().cuda_stream, x8.values.data_ptr(), w8.values.data_ptr(), x8.scales.data_ptr(), w8.scales.data_ptr()

    def call(rows=6, width=100, out=24, type=0, btype=0, act=3, x=X, ldx=128, xs=XS, w=W, ldw=128, ws=WS, yp=y.data_ptr(), ldy=24, r=None):
        return L.dgsp_linear_8bit(rows, width, out, type, btype, act, x, ldx, xs, w, ldw, ws, None, r, 24, yp, ldy, None, 0, stream)

    assert call() == dg.OK and call(rows=0, x=None, yp=None) == dg.OK
    assert call(rows=-1) == bad and call(width=0) == bad and call(out=0) == bad and call(type=4) == bad and call(btype=1) == bad and call(act=4) == bad
    assert call(x=None) == bad and call(xs=None) == bad and call(w=None) == bad and call(ws=None) == bad and call(yp=None) == bad
    assert call(x=X + 8) == bad and call(xs=XS + 1) == bad and call(ldx=96) == bad and call(ldw=136) == bad and call(ldy=23) == bad and call(ldx=1 << 23) == bad
    assert call(rows=1 << 31) == bad and call(width=1 << 22) == bad
    need = L.dgsp_linear_8bit_workspace_bytes(65, 8192, 64)
    assert need > 0                                                  # split along the depth
    assert L.dgsp_linear_8bit(65, 8192, 64, 0, 0, 3, X, 8192, XS, W, 8192, WS, None, None, 0, y.data_ptr(), 64, y.data_ptr(), need - 1, stream) == bad
    torch.cuda.synchronize()


def test_sizes_without_a_gpu():
    L = layers.lib()
    for extents in ((-1, 8, 8), (1 << 31, 8, 8), (8, 0, 8), (8, 8, 0), (8, 1 << 22, 8), (8, 8, 1 << 62)):
        assert L.dgsp_linear_8bit_workspace_bytes(*extents) == 0
    assert 0 <= L.dgsp_linear_8bit_workspace_bytes(0, 8192, 64) <= L.dgsp_linear_8bit_workspace_bytes(100, 8192, 64)
