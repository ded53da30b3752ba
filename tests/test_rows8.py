"""Rows in 8 bits on the GPU against their definition: the same bits, as each step of it is exact but one rounding."""
import pytest
import torch

import rows8_reference as ref8
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def spread(rows, width, dtype, seed):
    """Numbers of many magnitudes: rows, blocks and elements that differ by factors of up to 2^12."""
    x = torch.randn((rows, width), generator=gen(seed), dtype=torch.float64)
    x *= 2.0 ** torch.randint(-6, 7, (rows, 1), generator=gen(seed + 1)).double()
    blocks = torch.randint(-3, 4, (rows, -(-width // 32)), generator=gen(seed + 2)).double().repeat_interleave(32, 1)[:, :width]
    return (x * 2.0 ** blocks).to(dtype)


def check(x, kind, on_gpu=None):
    got = layers.quantise(x.cuda() if on_gpu is None else on_gpu, kind)
    want, e = ref8.quantised(x.reshape(-1, x.shape[-1]), kind)
    values = got.values.cpu().double().reshape(want.shape)
    bad = torch.isnan(want)
    if kind == "e4m3":
        assert torch.equal(torch.isnan(values), bad)
    assert torch.equal(values[~bad], want[~bad])
    rows, blocks = e.shape
    bytes_ = got.scales.cpu().transpose(0, 1).reshape(rows, -1)
    whole = torch.full_like(bytes_, 127)
    whole[:, :blocks] = (e + 127).to(torch.uint8)
    if kind == "int8":
        whole[:, :blocks][bad.view(rows, blocks, 32).any(-1)] = 255
    assert torch.equal(bytes_, whole)
    stands = ref8.stands_for(x.reshape(-1, x.shape[-1]), kind)
    for to in TYPES:
        back = layers.dequantise(got, to)
        assert back.shape == x.shape and back.dtype == to
        assert torch.equal(back.cpu().double().nan_to_num(7.0), stands.float().to(to).view(x.shape).double().nan_to_num(7.0))
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 5), (7, 8), (130, 31), (129, 32), (64, 33), (5, 64), (9, 96), (3, 100), (66, 128), (5, 129), (4, 500),
                                        (3, 1001), (2, 2048), (2, 2049), (3, 8192), (1, 20000)])
def test_quantise_and_back(rows, width, dtype, kind):
    print("[case] quantise", rows, width, dtype, kind, flush=True)
    check(spread(rows, width, dtype, 3 * rows + width), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_ends_of_the_range(kind, dtype):
    """Zeros, the largest and the smallest numbers of the type, amax at the border of a scale and next to it, ties, infinities and NaN."""
    print("[case] ends", kind, dtype, flush=True)
    info = torch.finfo(dtype)
    most = ref8.MOST[kind]
    x = torch.randn((40, 96), generator=gen(1), dtype=torch.float64)
    x[0] = 0.0
    x[1, 32:64] = -0.0
    x[2, 5] = info.max
    x[3, 40] = -info.max
    x[4, 95] = 0.999 * info.max
    x[5] = info.tiny
    x[6] = info.smallest_normal * torch.randn(96, generator=gen(2), dtype=torch.float64) * 0.25
    x[7] *= 1e-30
    x[8, 3] = most
    x[9, 3] = most * (1 + info.eps)
    x[10, 3] = most * (1 - info.eps)
    x[11, :32], x[11, 31] = torch.arange(32).double() + 0.5, most                # ties of whole numbers
    x[12, :32], x[12, 31] = (torch.arange(32).double() + 16.5) * 8, most         # ties of e4m3: steps of 16 from 128 on, 8 from 64 on
    x[13, 7] = float("inf")
    x[14, 70] = float("-inf")
    x[15, 50] = float("nan")
    x[16, 0], x[16, 31] = float("nan"), info.max
    x[17] = float("nan")
    check(x.to(dtype), kind)


@pytest.mark.gpu
def test_orders_and_leading_axes():
    print("[case] orders", flush=True)
    x = spread(24, 100, torch.bfloat16, 5)
    want = layers.quantise(x.cuda())
    wide = torch.full((24, 150), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 7:107] = x.cuda()
    flat = torch.zeros(24 * 100 + 1, dtype=x.dtype, device="cuda")
    flat[1:] = x.cuda().reshape(-1)
    for view in (wide[:, 7:107], flat[1:].view(24, 100), x.cuda().t().contiguous().t(), x.cuda().view(2, 12, 100), torch._neg_view(-x.cuda())):
        got = layers.quantise(view)
        assert got.values.shape == (*view.shape[:-1], 128) and got.width == 100
        assert torch.equal(got.values.view(torch.uint8).view(24, 128), want.values.view(torch.uint8)) and torch.equal(got.scales, want.scales)
        assert torch.equal(layers.dequantise(got).view(24, 100), layers.dequantise(want))
    row = x[:1].cuda().expand(24, 100)
    assert torch.equal(layers.dequantise(layers.quantise(row)), layers.dequantise(layers.quantise(row.contiguous())))
    # values that lie otherwise: rows apart, at an odd address, one row repeated
    apart = torch.zeros((24, 200), dtype=torch.uint8, device="cuda")
    apart[:, 3:131] = want.values.view(torch.uint8)
    for values in (apart.view(torch.float8_e4m3fn)[:, 3:131], want.values.t().contiguous().t()):
        assert torch.equal(layers.dequantise(layers.Rows8(values, want.scales, 100)), layers.dequantise(want))
    one = layers.Rows8(want.values[:1].expand(24, 128), want.scales[:, :1].expand(1, 24, 4), 100)
    assert torch.equal(layers.dequantise(one), layers.dequantise(want)[:1].expand(24, 100))
    empty = layers.quantise(torch.empty((0, 40), device="cuda"), "int8")
    assert empty.values.shape == (0, 64) and empty.scales.shape == (1, 0, 4) and layers.dequantise(empty).shape == (0, 40)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_every_byte_reads_back_as_its_value(kind):
    print("[case] bytes", kind, flush=True)
    values = torch.arange(256, dtype=torch.uint8).view(8, 32)
    values = values.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8)
    scales = torch.full((1, 8, 4), 127, dtype=torch.uint8)
    scales[0, :, 0] = torch.tensor([0, 1, 2, 100, 127, 200, 230, 255], dtype=torch.uint8)
    got = layers.dequantise(layers.Rows8(values.cuda(), scales.cuda(), 32)).cpu().double()
    want = ref8.read(values, scales, 32)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)].float().double())


@pytest.mark.gpu
def test_refusals():
    print("[case] refusals", flush=True)
    x = torch.randn((6, 40), device="cuda")
    q = layers.quantise(x)
    Rows8 = layers.Rows8
    calls = {
        "unknown kind": lambda: layers.quantise(x, "e5m2"),
        "kind of another type": lambda: layers.quantise(x, ["e4m3"]),
        "on the host": lambda: layers.quantise(x.cpu()),
        "of doubles": lambda: layers.quantise(x.double()),
        "no axis": lambda: layers.quantise(x[0, 0]),
        "empty rows": lambda: layers.quantise(x[:, :0]),
        "with a gradient": lambda: layers.quantise(x.clone().requires_grad_(True)),
        "no rows in 8 bits": lambda: layers.dequantise(x),
        "of another type": lambda: layers.dequantise(q, torch.float64),
        "values of another type": lambda: layers.dequantise(Rows8(q.values.float(), q.scales, 40)),
        "values on the host": lambda: layers.dequantise(Rows8(q.values.cpu(), q.scales, 40)),
        "scales on the host": lambda: layers.dequantise(Rows8(q.values, q.scales.cpu(), 40)),
        "scales of another type": lambda: layers.dequantise(Rows8(q.values, q.scales.int(), 40)),
        "fewer scales": lambda: layers.dequantise(Rows8(q.values, q.scales[:, :5], 40)),
        "another width": lambda: layers.dequantise(Rows8(q.values, q.scales, 70)),
        "no width": lambda: layers.dequantise(Rows8(q.values, q.scales, 0)),
        "part of a block": lambda: layers.dequantise(Rows8(q.values[:, :40], q.scales, 40)),
    }
    for name, call in calls.items():
        with pytest.raises(dg.DgspError):
            call()
            pytest.fail(name)
    with torch.no_grad():
        layers.quantise(x.clone().requires_grad_(True))


@pytest.mark.gpu
def test_refusals_of_the_c_entry_points():
    print("[case] refusals in C", flush=True)
    L, x = layers.lib(), torch.randn((6, 40), device="cuda")
    values, scales = torch.empty((6, 64), dtype=torch.uint8, device="cuda"), torch.empty((6, 4), dtype=torch.uint8, device="cuda")
    stream, bad = torch.cuda.current_stream().cuda_stream, dg.ERR_INVALID_ARG

    def there(rows=6, width=40, type=0, kind=0, xp=x.data_ptr(), ldx=40, v=values.data_ptr(), ldv=64, s=scales.data_ptr()):
        return L.dgsp_quantise(rows, width, type, kind, xp, ldx, v, ldv, s, stream)

    def back(rows=6, width=40, type=0, kind=0, xp=x.data_ptr(), ldx=40, v=values.data_ptr(), ldv=64, s=scales.data_ptr()):
        return L.dgsp_dequantise(rows, width, type, kind, v, ldv, s, xp, ldx, stream)

    for call in (there, back):
        assert call() == dg.OK and call(rows=0, xp=None, v=None, s=None) == dg.OK
        assert call(rows=-1) == bad and call(width=0) == bad and call(type=3) == bad and call(kind=2) == bad and call(kind=-1) == bad
        assert call(xp=None) == bad and call(v=None) == bad and call(s=None) == bad and call(ldx=39) == bad and call(ldv=48) == bad
        assert call(ldv=72) == bad and call(v=values.data_ptr() + 8) == bad and call(s=scales.data_ptr() + 2) == bad and call(rows=1 << 31) == bad
    assert there(ldv=0) == bad and back(ldx=0) == bad
    torch.cuda.synchronize()


def test_reference_rounds_to_the_nearest_even():
    """The oracle itself, against torch's conversion and known ties."""
    v = torch.linspace(-448, 448, 4001, dtype=torch.float64)
    assert torch.equal(ref8.nearest_e4m3(v), v.float().to(torch.float8_e4m3fn).double())
    ties = torch.tensor([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0], dtype=torch.float64)
    assert ref8.nearest_e4m3(ties).tolist() == [16.0, 20.0, 0.0, 2.0 ** -8, 448.0]
    e = ref8.exponents(torch.tensor([[448.0], [449.0], [0.0], [1.0]]), "e4m3", torch.float32)
    assert e.view(-1).tolist() == [0, 1, 0, -8]
