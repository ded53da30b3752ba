"""Performance cases of the layers around a sparse product: layer norm, dropout and the gated feed-forward block.

A graph network's layer multiplies by the sparse matrix and then works on the dense features, rows x width, one row per
vertex (or per token): the sum with the residual, its normalisation, a feed-forward block, dropout.  A case is a dict of
plain values:
  op      "layer_norm"      y = (x - mean) / sqrt(var + eps) * weight + bias, over the last axis
          "add_layer_norm"  s = residual + dropout(x), y = the layer norm of s; both are results
          "dropout"         y = dropout(x), or residual + dropout(x)
          "gated_ff"        y = (act(x Wg^T) * (x Wu^T)) Wd^T
  rows, width, hidden   x is rows x width; Wg and Wu are hidden x width, Wd is width x hidden
  dtype   of inputs and results: "fp32", "bf16", "fp16"; `params`: of the norm's weight and bias
  train   results and gradients (of all inputs and parameters), or results alone
  p, act, residual      drop rate; "silu", "gelu" (by the error function), "relu"; is there a residual

Dropout's random numbers are a function of seed and offset, which are inputs.  Element (row, col) is kept where a 16-bit number
is at least round(65536 p), and then scaled by 65536 / (65536 - round(65536 p)).  The number is the (col % 8)-th of the eight that
Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw, SC 2011) makes of the counter (col // 8, row, offset's low word, its high
word) and the key (seed's low word, its high word), lower halves first.

All inputs are made on the GPU from the seed alone.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
ACTIVATIONS = ("silu", "gelu", "relu")

# what no drawn case exceeds
MOST_NORM = 1 << 26
MOST_DROPOUT = 1 << 27
MOST_HIDDEN = 1 << 27
MOST_FLOPS = {"bf16": 9.8e12, "fp16": 9.8e12, "fp32": 1.5e12}


def _norm(name, rows, width, dtype, train, params=None):
    return dict(name=name, op="layer_norm", rows=rows, width=width, dtype=dtype, params=params or dtype, train=train)


def _add_norm(name, rows, width, dtype, p, train, params=None):
    return dict(name=name, op="add_layer_norm", rows=rows, width=width, dtype=dtype, params=params or dtype, p=p, train=train)


def _dropout(name, rows, width, dtype, p, residual, train):
    return dict(name=name, op="dropout", rows=rows, width=width, dtype=dtype, p=p, residual=residual, train=train)


def _gated(name, rows, width, hidden, dtype, act, train):
    return dict(name=name, op="gated_ff", rows=rows, width=width, hidden=hidden, dtype=dtype, act=act, train=train)


def listed():
    return [
        # one token or vertex in a serving loop: the launch and the host are all of it
        _norm("norm_token", 1, 4096, "bf16", False),
        # training on a graph of 2^20 vertices at the benchmark's feature width 32: rows far shorter than a wave can read
        _norm("norm_graph_train", 1 << 20, 32, "fp32", True),
        # training on long sequences with a large width, parameters kept in 32 bits
        _norm("norm_wide_train", 8192, 8192, "bf16", True, params="fp32"),
        # a residual block's sum, dropout and normalisation in a training step
        _add_norm("add_norm_train", 32768, 1024, "bf16", 0.1, True),
        # the same at odd sizes throughout: a batch of sampled vertices, a width that no vector divides
        _add_norm("add_norm_odd_train", 4099, 1001, "fp16", 0.25, True),
        # the benchmark's smallest features, 4096 x 4
        _dropout("dropout_tiny", 4096, 4, "fp32", 0.5, False, False),
        # features of 2^20 vertices at the benchmark's largest width: dropout onto the residual, with its gradient
        _dropout("dropout_graph_train", 1 << 20, 128, "bf16", 0.1, True, True),
        # one token through a large block: every weight is read for it
        _gated("gated_token", 1, 4096, 16384, "bf16", "silu", False),
        # a small batch with odd sizes throughout
        _gated("gated_batch_odd", 37, 1000, 2731, "fp16", "gelu", False),
        # training on a graph of 2^20 vertices at width 64: features are many, weights are few
        _gated("gated_graph_train", 1 << 20, 64, 128, "bf16", "silu", True),
        # training on a graph of 2^16 vertices in the sparse product's own type
        _gated("gated_fp32_train", 1 << 16, 128, 512, "fp32", "gelu", True),
        # training step of a large block on 8192 tokens
        _gated("gated_train", 8192, 4096, 16384, "bf16", "silu", True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operator, type and direction at random, sizes over the listed ranges."""
    while True:
        op = rng.choice(("layer_norm", "add_layer_norm", "dropout", "gated_ff"))
        dtype, train = rng.choice(("fp32", "bf16", "fp16")), rng.random() < 0.6
        rows = _log_between(rng, 1, 1 << 20)
        case = dict(op=op, rows=rows, dtype=dtype, train=train)
        if rows == 3072:                                # sizes that no program here has
            continue
        if op == "gated_ff":
            width, hidden = _log_between(rng, 16, 4096), _log_between(rng, 32, 16384)
            if rng.random() < 0.5:                      # half of the programs choose multiples of 16
                width, hidden = -(-width // 16) * 16, -(-hidden // 16) * 16
            case.update(width=width, hidden=hidden, act=rng.choice(ACTIVATIONS))
            if 3072 not in (width, hidden) and rows * max(width, hidden) <= MOST_HIDDEN and 18.0 * rows * width * hidden <= MOST_FLOPS[dtype]:
                return case
            continue
        width = _log_between(rng, 4, 8192)
        if rng.random() < 0.5:
            width = -(-width // 8) * 8
        case["width"] = width
        if op != "dropout":
            case["params"] = rng.choice((dtype, "fp32"))
        else:
            case["residual"] = rng.random() < 0.5
        if op != "layer_norm":
            case["p"] = rng.choice((0.0, 0.05, 0.1, 0.25, 0.5))
        if width != 3072 and rows * width <= (MOST_DROPOUT if op == "dropout" else MOST_NORM):
            return case


# ---------------------------------------------------------------------------------------------- inputs

def _features(rows, width, gen):
    """Columns with means and scales of their own, a few of them much larger than the rest."""
    scale = torch.exp(torch.randn(width, device="cuda", generator=gen) * 0.3)
    scale[torch.rand(width, device="cuda", generator=gen) < 0.01] *= 10.0
    x = torch.randn((rows, width), device="cuda", generator=gen)
    return x.add_(torch.randn(width, device="cuda", generator=gen), alpha=0.5).mul_(scale)


def _inputs(case, seed):
    """Inputs by name, in the case's types, and the gradient of each result."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, width, dtype, op = case["rows"], case["width"], DTYPES[case["dtype"]], case["op"]
    given, grads = {}, {}

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if op == "gated_ff":
        hidden = case["hidden"]
        given["x"] = normal(rows, width).to(dtype)
        given["w_gate"] = normal(hidden, width).mul_(width ** -0.5).to(dtype)
        given["w_up"] = normal(hidden, width).mul_(width ** -0.5).to(dtype)
        given["w_down"] = normal(width, hidden).mul_(hidden ** -0.5).to(dtype)
    else:
        given["x"] = _features(rows, width, gen).to(dtype)
        if op == "add_layer_norm" or case.get("residual"):
            given["residual"] = _features(rows, width, gen).to(dtype)
        if op != "dropout":
            given["weight"] = normal(width).mul_(0.1).add_(1.0).to(DTYPES[case["params"]])
            given["bias"] = normal(width).mul_(0.1).to(DTYPES[case["params"]])
    if case["train"]:
        grads["y"] = normal(rows, width).to(dtype)
        if op == "add_layer_norm":
            grads["s"] = normal(rows, width).to(dtype)
    return given, grads


def _drop_key(seed):
    """What a program's dropout layer holds: its seed and the number of the call."""
    return (seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 64), (seed * 77 + (1 << 33) + 5) % (1 << 40)


def prepare(case, seed):
    given, grads = _inputs(case, seed)
    drop_seed, drop_offset = _drop_key(seed)
    if case["train"]:
        for t in given.values():
            t.requires_grad_(True)
    return dict(case=case, given=given, grads=grads, seed=drop_seed, offset=drop_offset)


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2106_16064_amd import layers
    case, given = state["case"], state["given"]
    op, p = case["op"], case.get("p", 0.0)
    with torch.set_grad_enabled(case["train"]):
        if op == "layer_norm":
            results = {"y": layers.layer_norm(given["x"], given["weight"], given["bias"], eps=EPS)}
        elif op == "add_layer_norm":
            y, s = layers.add_layer_norm(given["x"], given["residual"], given["weight"], given["bias"], eps=EPS, p=p,
                                         seed=state["seed"], offset=state["offset"])
            results = {"y": y, "s": s}
        elif op == "dropout":
            results = {"y": layers.dropout(given["x"], p, state["seed"], state["offset"], residual=given.get("residual"))}
        else:
            results = {"y": layers.gated_ff(given["x"], given["w_gate"], given["w_up"], given["w_down"], activation=case["act"])}
        out = {k: t.detach() for k, t in results.items()}
        if case["train"]:
            grads = torch.autograd.grad([results[k] for k in state["grads"]], list(given.values()), list(state["grads"].values()))
            out.update({"d_" + k: g for k, g in zip(given, grads)})
    return out


# ---------------------------------------------------------------------------------------------- the plain forms

def _philox_halves(rows, width, seed, offset):
    """rows x width numbers of 16 bits, as the module's text defines them, on the GPU."""
    low = 0xFFFFFFFF
    groups = -(-width // 8)
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c2 = torch.full((), offset & low, device="cuda", dtype=torch.int64).expand(rows, groups)
    c3 = torch.full((), offset >> 32, device="cuda", dtype=torch.int64).expand(rows, groups)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # 64-bit products, modulo 2^64
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((c0, c1, c2, c3), dim=-1)
    return torch.stack((words & 0xFFFF, words >> 16), dim=-1).reshape(rows, groups * 8)[:, :width]


def _keep_scale(case, state):
    """What each element is multiplied by: 0 or the scale."""
    dropped = math.floor(case["p"] * 65536 + 0.5)
    keep = _philox_halves(case["rows"], case["width"], state["seed"], state["offset"]) >= dropped
    return keep.float() * (65536.0 / (65536 - dropped) if dropped < 65536 else 0.0)


def _act(kind, g):
    """act(g) and its derivative."""
    if kind == "relu":
        return g.clamp(min=0.0), (g > 0).float()
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    c = 0.5 * (1.0 + torch.erf(g * (0.5 ** 0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * ((2.0 * math.pi) ** -0.5)


def _run_plain(state):
    case, given, dtype = state["case"], state["given"], DTYPES[state["case"]["dtype"]]
    op = case["op"]
    with torch.no_grad():
        x = given["x"].float()
        g = {k: t.float() for k, t in state["grads"].items()}
        out = {}
        if op == "gated_ff":
            wg, wu, wd = (given[k].float() for k in ("w_gate", "w_up", "w_down"))
            gate, up = x @ wg.t(), x @ wu.t()
            act, slope = _act(case["act"], gate)
            h = act * up
            out["y"] = h @ wd.t()
            if case["train"]:
                dh = g["y"] @ wd
                dg, du = dh * up * slope, dh * act
                out["d_x"] = dg @ wg + du @ wu
                out["d_w_gate"], out["d_w_up"], out["d_w_down"] = dg.t() @ x, du.t() @ x, g["y"].t() @ h
            return {k: t.to(dtype) for k, t in out.items()}

        scale = _keep_scale(case, state) if op != "layer_norm" else None
        s = x if scale is None else x * scale
        if "residual" in given:
            s = s + given["residual"].float()
        if op == "dropout":
            out["y"] = s
            if case["train"]:
                out["d_x"] = g["y"] * scale
                if "residual" in given:
                    out["d_residual"] = g["y"]
            return {k: t.to(dtype) for k, t in out.items()}

        w, b = given["weight"].float(), given["bias"].float()
        centred = s - s.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
        hat = centred * rstd
        out["y"] = hat * w + b
        if op == "add_layer_norm":
            out["s"] = s
        if case["train"]:
            dhat = g["y"] * w
            ds = (dhat - dhat.mean(1, keepdim=True) - hat * (dhat * hat).mean(1, keepdim=True)) * rstd
            if op == "add_layer_norm":
                ds = ds + g["s"]
                out["d_x"], out["d_residual"] = ds * scale, ds
            else:
                out["d_x"] = ds
            out["d_weight"], out["d_bias"] = (g["y"] * hat).sum(0), g["y"].sum(0)
        params = DTYPES[case["params"]]
        return {k: t.to(params if k in ("d_weight", "d_bias") else dtype) for k, t in out.items()}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _kept_64(rows, width, p, seed, offset):
    """The multipliers of dropout in 64 bits, from the generator's definition in whole numbers on the host."""
    mask, halves = np.uint64(0xFFFFFFFF), []
    groups = -(-width // 8)
    step = max(1, (1 << 21) // groups)
    for first in range(0, rows, step):
        last = min(rows, first + step)
        n = last - first
        c = [np.tile(np.arange(groups, dtype=np.uint64), n), np.repeat(np.arange(first, last, dtype=np.uint64), groups),
             np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32)]
        key = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), p1 & mask, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), p0 & mask]
            key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
        words = np.stack([np.broadcast_to(w, (n * groups,)) for w in c], axis=1).astype("<u4")
        halves.append(np.ascontiguousarray(words).view("<u2").reshape(n, groups * 8)[:, :width])
    dropped = int(math.floor(p * 65536 + 0.5))
    keep = torch.from_numpy(np.concatenate(halves) >= dropped).cuda()
    return keep.double() * (65536.0 / (65536 - dropped) if dropped < 65536 else 0.0)


def exact(case, seed):
    """The forward definitions in 64 bits; gradients by differentiating those."""
    given, grads = _inputs(case, seed)
    leaf = {k: t.double().requires_grad_(case["train"]) for k, t in given.items()}
    op = case["op"]
    results = {}
    with torch.set_grad_enabled(case["train"]):
        if op == "gated_ff":
            gate = torch.nn.functional.linear(leaf["x"], leaf["w_gate"])
            act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[case["act"]]
            hidden = act(gate) * torch.nn.functional.linear(leaf["x"], leaf["w_up"])
            results["y"] = torch.nn.functional.linear(hidden, leaf["w_down"])
        else:
            s = leaf["x"]
            if op != "layer_norm":
                s = s * _kept_64(case["rows"], case["width"], case["p"], *_drop_key(seed))
            if "residual" in leaf:
                s = s + leaf["residual"]
            if op == "dropout":
                results["y"] = s
            else:
                var, mean = torch.var_mean(s, dim=1, unbiased=False, keepdim=True)
                results["y"] = leaf["weight"] * (s - mean) * torch.rsqrt(var + EPS) + leaf["bias"]
                if op == "add_layer_norm":
                    results["s"] = s
        out = {k: t.detach() for k, t in results.items()}
        if case["train"]:
            wrt = torch.autograd.grad([results[k] for k in grads], list(leaf.values()), [t.double() for t in grads.values()])
            out.update({"d_" + k: t for k, t in zip(leaf, wrt)})
    return out


# ---------------------------------------------------------------------------------------------- what it costs at least

def work(case):
    rows, width, size, op = case["rows"], case["width"], BYTES[case["dtype"]], case["op"]
    n, train = rows * width, case["train"]
    if op == "gated_ff":
        hidden = case["hidden"]
        weights = 3 * width * hidden
        return {"bytes": size * ((4 if train else 2) * n + (2 if train else 1) * weights),
                "flops": (18 if train else 6) * n * hidden}
    passes = 2                                            # x, y
    if train:
        passes += 2                                       # dy, dx
    if op == "add_layer_norm":
        passes += 2 + (2 if train else 0)                 # residual, s; ds, d_residual
    elif case.get("residual"):
        passes += 1                                       # residual; its gradient is dy itself
    params = 0 if op == "dropout" else BYTES[case["params"]] * width * (4 if train else 2)
    per = {"layer_norm": 8, "add_layer_norm": 12, "dropout": 3}[op] + ((12 if op != "dropout" else 2) if train else 0)
    return {"bytes": size * passes * n + params, "flops": per * n}
