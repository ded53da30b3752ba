"""The product and its gradient of -1, 0 and 1, without an activation or with relu: all sums are whole numbers below 2^24, which 32 bits hold whatever
the order, x in 8 bits stands for itself, and each result is that of 64 bits, rounded once.  A row, a column or a part of a sum that is left out
or counted twice shows, however many there are."""
import pytest
import torch

from paper_2106_16064_amd import layers
from test_linear import check, inputs

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def digits(shape, dtype, seed):
    return torch.randint(-1, 2, shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed), dtype=torch.int8).to(dtype)


def check_exact(rows, width, out, dtype, params, kind, keep, residual=True):
    """Both passes; the definition goes over the rows in pieces."""
    print("[case] exact", rows, width, out, dtype, params, kind, keep, flush=True)
    x, w, dy = digits((rows, width), dtype, 0), digits((out, width), dtype, 1), digits((rows, out), dtype, 2)
    b, r = digits((out,), params, 3), digits((rows, out), dtype, 4) if residual else None
    leaves = [t.requires_grad_(True) for t in (x, w, b)]
    y = layers.linear(*leaves, kind, r, keep)
    dx, dw, db = torch.autograd.grad(y, leaves, dy)
    y = y.detach()
    W, B = w.detach().double(), b.detach().double()
    want_w, want_b = torch.zeros((out, width), dtype=torch.float64, device="cuda"), torch.zeros(out, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // max(width, out))
    for first in range(0, rows, step):
        part = slice(first, min(rows, first + step))
        X, G = x.detach()[part].double(), dy[part].double()
        z = X @ W.t() + B
        value = z.clamp(min=0) if kind == "relu" else z
        assert torch.equal(y[part], (value if r is None else value + r[part].double()).to(dtype)), "y"
        dz = G * (z > 0) if kind == "relu" else G
        assert torch.equal(dx[part], (dz @ W).to(dtype)), "dx"
        want_w += dz.t() @ X
        want_b += dz.sum(0)
    assert torch.equal(dw, want_w.to(dtype)), "dweight"
    assert torch.equal(db, want_b.to(params)), "dbias"


NARROW = [(width, out) for width in (32, 64, 128) for out in (32, 64, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,out", NARROW)
def test_whole_narrow_rows(width, out, dtype):
    """Widths that are exactly 32, 64 or 128 have kernels of their own; more rows than the workgroups take in one turn, and no whole tiles of them."""
    for params in {dtype, torch.float32}:
        for kind in (None, "relu"):
            for keep in (False, True):
                check_exact(70001, width, out, dtype, params, kind, keep, residual=kind is None)
    check_exact(200003, width, out, dtype, dtype, "relu", True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("width,out", NARROW)
def test_whole_narrow_rows_against_64_bits(width, out, dtype, kind):
    for rows in (203, 50):
        print("[case] whole narrow rows", rows, width, out, dtype, kind, flush=True)
        for params in {dtype, torch.float32}:
            for keep in (False, True):
                x, w, b, r, dy = inputs(rows, width, out, dtype, params, 400)
                check((x, w, b, r if keep else None, dy), kind, keep)
        x, w, b, r, dy = inputs(rows, width, out, dtype, dtype, 410)
        check((x, w, None, r, dy), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,width,out", [((1 << 20) + 77, 40, 2056), ((1 << 20) + 77, 2056, 24), ((1 << 25) + 77, 64, 72), ((1 << 25) + 77, 64, 64)])
def test_gradients_of_more_than_2_to_the_31_elements(rows, width, out, dtype, keep):
    check_exact(rows, width, out, dtype, torch.float32, "relu", keep)


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,out", [(8192, 4096, 16384), (8185, 4100, 4104), (50000, 301, 777), (16384, 1024, 4096), (65537, 128, 512), (131079, 33, 70)])
def test_large_products(rows, width, out, dtype, keep):
    if keep and rows == 8192:
        return check_exact(2048, width, out, dtype, dtype, None, keep)
    check_exact(rows, width, out, dtype, dtype, "relu", keep)
