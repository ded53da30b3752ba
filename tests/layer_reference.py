"""The layers from their definitions, in 64 bits on the host, for the tests."""
import math

import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step at 1
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}                  # half of the smallest step
EPS32 = 2.0 ** -24


def philox(c, k):
    """Philox4x32 with 10 rounds on whole numbers: counter and key are sequences of integers below 2^32."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def halves(rows, width, seed, offset):
    """The 16-bit numbers of rows x width elements."""
    m = np.uint64(0xFFFFFFFF)
    s32 = np.uint64(32)
    groups = -(-width // 8)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), groups),
         np.full(rows * groups, offset & 0xFFFFFFFF, dtype=np.uint64), np.full(rows * groups, offset >> 32, dtype=np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s32) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    out = np.empty((rows * groups, 8), dtype=np.int64)
    for i in range(4):
        out[:, 2 * i] = (c[i] & np.uint64(0xFFFF)).astype(np.int64)
        out[:, 2 * i + 1] = (c[i] >> np.uint64(16)).astype(np.int64)
    return out.reshape(rows, groups * 8)[:, :width]


def keep_scale(rows, width, p, seed, offset):
    """The kept elements (bool) and their multiplier."""
    t = math.floor(p * 65536 + 0.5)
    return torch.from_numpy(halves(rows, width, seed, offset) >= t), (65536.0 / (65536 - t) if t < 65536 else 0.0)


def dropped(x, p, seed, offset):
    keep, scale = keep_scale(*x.shape, p, seed, offset)
    return torch.where(keep, x * scale, torch.zeros((), dtype=x.dtype))


def norm(s, weight, bias, eps):
    mean = s.mean(1, keepdim=True)
    var = ((s - mean) ** 2).mean(1, keepdim=True)
    y = (s - mean) / torch.sqrt(var + eps)
    if weight is not None:
        y = y * weight
    return y + bias if bias is not None else y


def act(kind, g):
    if kind == "relu":
        return torch.where(g > 0, g, torch.zeros((), dtype=g.dtype))
    if kind == "silu":
        return g / (1 + torch.exp(-g))
    return g * 0.5 * (1 + torch.erf(g / math.sqrt(2.0)))


def slope(kind, g):
    if kind == "relu":
        return (g > 0).to(g.dtype)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s + g * s * (1 - s)
    return 0.5 * (1 + torch.erf(g / math.sqrt(2.0))) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def norm_gradient(s, weight, dy, eps):
    """Gradients of s, of the weight and of the bias, by the formula."""
    mean = s.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + eps)
    hat = (s - mean) * rstd
    dhat = dy if weight is None else dy * weight
    ds = (dhat - dhat.mean(1, keepdim=True) - hat * (dhat * hat).mean(1, keepdim=True)) * rstd
    return ds, (dy * hat).sum(0), dy.sum(0)


def assert_within(got, want, bound, what):
    """|got - want| <= bound for every element; what is not finite has to agree in kind."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~torch.isfinite(want)
    assert bool((torch.isnan(got[bad]) == torch.isnan(want[bad])).all()), what
    over = (got - want).abs()[~bad] - bound.expand_as(want)[~bad]
    if over.numel():
        worst = float(over.max())
        assert worst <= 0, f"{what}: {worst:.3e} beyond the bound ({int((over > 0).sum())} of {over.numel()} elements)"
