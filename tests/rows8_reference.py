"""Rows in 8 bits from their definition, in 64 bits on the host, for the tests."""
import torch

MOST = {"e4m3": 448.0, "int8": 127.0}


def exponents(x, kind, dtype):
    """[rows][blocks] of the least e with amax <= most 2^e, found by trying all of them."""
    blocks = cut(x).abs()
    amax = torch.where(torch.isfinite(blocks), blocks, torch.zeros((), dtype=torch.float64)).amax(-1)
    least, most = (-24, 9) if kind == "int8" and dtype == torch.float16 else (-126, 119 if kind == "e4m3" else 121)
    e = torch.full(amax.shape, most)
    for k in range(most - 1, least - 1, -1):
        e = torch.where(amax <= MOST[kind] * 2.0 ** k, torch.full((), k), e)
    return torch.where(amax == 0, torch.zeros((), dtype=e.dtype), e)


def cut(x):
    rows, width = x.shape
    filled = torch.zeros((rows, -(-width // 32) * 32), dtype=torch.float64)
    filled[:, :width] = x.double()
    return filled.view(rows, -1, 32)


def e4m3_values():
    """Every finite number of the format, ascending."""
    found = {0.0}
    for exponent in range(16):
        for fraction in range(8):
            if (exponent, fraction) == (15, 7):
                continue                                                 # NaN
            v = fraction / 8 * 2.0 ** -6 if exponent == 0 else (1 + fraction / 8) * 2.0 ** (exponent - 7)
            found |= {v, -v}
    return torch.tensor(sorted(found), dtype=torch.float64)


def nearest_e4m3(v):
    """The nearest of them, ties to the one whose last bit is 0: of two neighbours the one with the even place in the order from 0 on."""
    table = e4m3_values()
    zero = len(table) // 2
    flat = v.reshape(-1).clamp(-448.0, 448.0)
    at = torch.searchsorted(table, flat).clamp(1, len(table) - 1)
    low, high = table[at - 1], table[at]
    up = (high - flat < flat - low) | ((high - flat == flat - low) & ((at - zero) % 2 == 0))
    return torch.where(up, high, low).view(v.shape)


def quantised(x, kind):
    """(elements over their scales [rows][32 blocks], exponents [rows][blocks]; NaN where a block or element is none)."""
    e = exponents(x, kind, x.dtype)
    v = cut(x) / 2.0 ** e.double()[..., None]
    bad = ~torch.isfinite(v)
    if kind == "e4m3":
        out = torch.where(bad, torch.full((), float("nan"), dtype=torch.float64), nearest_e4m3(torch.where(bad, torch.zeros((), dtype=torch.float64), v)))
    else:
        out = torch.where(bad, torch.zeros((), dtype=torch.float64), torch.round(v).clamp(-127, 127))
        out = torch.where(bad.any(-1, keepdim=True), torch.full((), float("nan"), dtype=torch.float64), out)
    return out.reshape(x.shape[0], -1), e


def stands_for(x, kind):
    """x as rows in 8 bits stand for it."""
    v, e = quantised(x, kind)
    return (v.view(x.shape[0], -1, 32) * 2.0 ** e.double()[..., None]).reshape(x.shape[0], -1)[:, :x.shape[1]]


def read(values, scales, width):
    """What values and scales, as they are laid out, stand for; from their bytes."""
    rows = values.reshape(-1, values.shape[-1]).shape[0]
    blocks = -(-width // 32)
    assert values.shape[-1] == 32 * blocks and scales.shape == (-(-blocks // 4), rows, 4) and scales.dtype == torch.uint8
    v = values.cpu().reshape(rows, blocks, 32).double()
    b = scales.cpu().transpose(0, 1).reshape(rows, -1)
    assert bool((b[:, blocks:] == 127).all())
    b = b[:, :blocks].double()
    factor = torch.where(b == 255, torch.full((), float("nan"), dtype=torch.float64), 2.0 ** (b - 127))
    full = (v * factor[..., None]).reshape(rows, -1)
    assert bool((v.reshape(rows, -1)[:, width:] == 0).all())
    return full[:, :width]
