"""Performance cases of the operators beside the optimizer: what a layer of a torch model runs when the n workers'
micro-batches go through it as one batch, worker by worker along the leading axis, with each worker's weight gradients kept
apart as the rows that COMP-AMS compresses.

    dropout                  x [n, rows, h]; the mask comes from a counter-based generator and is never stored
    layer_norm               forward, and backward with the weight's gradient of every worker
    dropout_add_layer_norm   the branch's dropout, the residual sum and the norm that follows, as one operator
    low_rank_adapter         base + scale (dropout(x) A^T) B^T beside a projection that is not trained

The mask. Element c of row j of worker i is kept where a 16-bit number u >= round(65536 p); kept values are multiplied by
65536 / (65536 - round(65536 p)). u is a half of a word of the Philox4x32-10 block (Salmon, Moraes, Dror, Shaw, SC 2011) at
counter (c // 8, j, i, call) under key (seed mod 2^32, seed div 2^32): word (c % 8) // 2, its low half where c is even.

"infer" passes run forward, "train" passes forward and backward. fp32 parameters throughout, as the optimizer keeps them.
"""
from __future__ import annotations

import functools
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = 1 << 27  # elements of one activation


def case(name, op, mode, dtype, n, rows, h, out=0, rank=0, p=0.0, shared=True, residual=""):
    c = {"op": op, "mode": mode, "dtype": dtype, "n": n, "rows": rows, "h": h, "out": out, "rank": rank, "p": p,
         "shared": shared, "residual": residual or dtype}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # activations of eight workers' micro-batches in mixed precision
        case("dropout bf16 n=8 h=4096", "dropout", "train", "bf16", 8, 2048, 4096, p=0.1),
        # a full-precision model with an odd width
        case("dropout f32 n=4 h=1001", "dropout", "train", "f32", 4, 513, 1001, p=0.5),
        # one token while answering: latency
        case("norm one token h=4096", "layer_norm", "infer", "bf16", 1, 1, 4096),
        # sixteen workers with small full-precision micro-batches
        case("norm f32 n=16 h=512", "layer_norm", "train", "f32", 16, 128, 512),
        # eight workers with long micro-batches in mixed precision
        case("norm bf16 n=8 h=4096", "layer_norm", "train", "bf16", 8, 2048, 4096),
        # an odd width in half precision, every row on another boundary
        case("norm f16 n=3 h=1001", "layer_norm", "train", "f16", 3, 777, 1001),
        # the end of a transformer's branch, the largest activation here
        case("add norm bf16 n=8 h=4096", "dropout_add_layer_norm", "train", "bf16", 8, 4096, 4096, p=0.1),
        # the residual stream kept in full precision, ragged micro-batches
        case("add norm bf16/f32 n=16 h=1000", "dropout_add_layer_norm", "train", "bf16", 16, 333, 1000, p=0.1, residual="f32"),
        # one token of each of 32 requests, every request with an adapter of its own
        case("adapter 32 tokens r=16", "low_rank_adapter", "infer", "bf16", 32, 1, 4096, out=4096, rank=16, shared=False),
        # fine-tuning: eight workers train one adapter
        case("adapter bf16 n=8 r=16", "low_rank_adapter", "train", "bf16", 8, 512, 4096, out=4096, rank=16, p=0.05),
        # a small full-precision model with odd widths
        case("adapter f32 n=4 r=8", "low_rank_adapter", "train", "f32", 4, 300, 1000, out=777, rank=8, p=0.1),
        # long micro-batches, a wide projection, a high rank
        case("adapter bf16 n=8 r=64", "low_rank_adapter", "train", "bf16", 8, 2048, 4096, out=8192, rank=64, p=0.1),
    ]


def _spread(rng, low, high):
    """A size between the two, evenly over its logarithm; as a rule, but not always, a multiple of 8."""
    v = int(math.exp(rng.uniform(math.log(low), math.log(high + 1.0))))
    return v if v < 16 or rng.random() < 0.4 else v // 8 * 8


def draw(rng: random.Random):
    op = rng.choice(["dropout", "layer_norm", "dropout_add_layer_norm", "low_rank_adapter"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    mode = "train" if op == "dropout" or rng.random() < 0.7 else "infer"
    n, rows, h = _spread(rng, 1, 32), _spread(rng, 1, 8192), _spread(rng, 8, 16384)
    p = 0.0 if mode == "infer" or op == "layer_norm" else rng.choice([0.0, 0.05, 0.1, 0.25, 0.5])
    if op == "dropout":
        p = max(p, 0.05)
    out = rank = 0
    residual = rng.choice([dtype, "f32"]) if op == "dropout_add_layer_norm" else dtype
    if op == "low_rank_adapter":
        out, rank = _spread(rng, 8, 16384), rng.choice([1, 2, 4, 8, 8, 12, 16, 16, 24, 32, 64, 128])
    most = LARGEST if op != "low_rank_adapter" else LARGEST // 2 * 16 // max(16, rank)
    while n * rows * max(h, out) > most // (2 if "f32" in (dtype, residual) else 1):
        rows = rows // 2 + rng.randrange(2) if rows > 2 else 1
        n = n if rows > 1 else max(1, n // 2)
    return case("", op, mode, dtype, n, rows, h, out, rank, p, rng.random() < 0.7, residual)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t, n, rows, h = TYPES[case["dtype"]], case["n"], case["rows"], case["h"]

    def normal(*shape, sigma=1.0, dtype=torch.float32):
        return (sigma * torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)).to(dtype)

    # the generator's key and this call's number, as a training program counts them
    s = {"case": case, "seed": (int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), "call": int(seed) % 1000 + 1}
    if case["op"] == "low_rank_adapter":
        out, r = case["out"], case["rank"]
        many = 1 if case["shared"] else n
        s["x"], s["base"] = normal(n, rows, h, dtype=t), normal(n, rows, out, dtype=t)
        s["A"], s["B"] = normal(many, r, h, sigma=h ** -0.5).expand(n, r, h), normal(many, out, r, sigma=r ** -0.5).expand(n, out, r)
        s["scale"] = 2.0
        if case["mode"] == "train":
            s["dy"] = normal(n, rows, out, sigma=0.02, dtype=t)
        return s
    # activations: channels of different sizes, each off zero by a little
    s["x"] = (normal(n, rows, h) * (0.5 + normal(h).abs()) + 0.1 * normal(h)).to(t)
    if case["mode"] == "train":
        s["dy"] = normal(n, rows, h, sigma=0.02, dtype=t)
    if case["op"] == "dropout":
        return s
    # one weight for all workers, seen by each of them: its gradient is kept apart by worker
    s["weight"], s["bias"] = (1.0 + 0.2 * normal(h)).expand(n, h), (0.2 * normal(h)).expand(n, h)
    s["eps"] = 1e-5
    if case["op"] == "dropout_add_layer_norm":
        s["residual"] = normal(n, rows, h, sigma=2.0, dtype=TYPES[case["residual"]])
        if case["mode"] == "train":
            s["ds"] = normal(n, rows, h, sigma=0.02, dtype=TYPES[case["residual"]])
    return s


# ---- the operators in their plain form ------------------------------------------------------------------------------------


def _wide_product(a, x):
    """High and low 32 bits of a x, for 32-bit numbers held in int64."""
    low, high = a * (x & 0xFFFF), a * (x >> 16)
    return (high + (low >> 16)) >> 16, (((high & 0xFFFF) << 16) + low) & 0xFFFFFFFF


def _round(c, key):
    h0, l0 = _wide_product(0xD2511F53, c[0])
    h1, l1 = _wide_product(0xCD9E8D57, c[2])
    return h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0


def _threshold(p):
    return int(math.floor(65536.0 * p + 0.5))


def _keep(state, n, rows, h):
    """The mask [n, rows, h]."""
    seed, groups = state["seed"], (h + 7) // 8
    keys = [((seed + r * 0x9E3779B9) & 0xFFFFFFFF, ((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF) for r in range(10)]
    at = functools.partial(torch.arange, device="cuda", dtype=torch.int64)
    counter = (at(groups)[None, None], at(rows)[None, :, None], at(n)[:, None, None],
               torch.full((1, 1, 1), state["call"], device="cuda", dtype=torch.int64))
    words = torch.stack(functools.reduce(_round, keys, counter), dim=-1)
    u = torch.stack((words & 0xFFFF, words >> 16), dim=-1).reshape(n, rows, 8 * groups)[:, :, :h]
    return u >= _threshold(state["case"]["p"])


def _dropped(v, state):
    """Dropout of fp32 values [n, rows, h]; its own gradient as well."""
    p = state["case"]["p"]
    if p == 0.0:
        return v
    t = _threshold(p)
    return torch.where(_keep(state, *v.shape), v * (65536.0 / (65536 - t)), torch.zeros_like(v))


def _norm(v, weight, bias, eps):
    mean = v.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v - mean).square().mean(-1, keepdim=True) + eps)
    xhat = (v - mean) * rstd
    return xhat * weight[:, None] + bias[:, None], xhat, rstd


def _norm_gradients(dy, xhat, rstd, weight):
    g = dy * weight[:, None]
    dv = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return dv, (dy * xhat).sum(1), dy.sum(1)


def _plain(state):
    case = state["case"]
    op, t, train = case["op"], TYPES[case["dtype"]], case["mode"] == "train"
    x = state["x"].float()
    if op == "dropout":
        y = _dropped(x, state).to(t)
        return {"y": y, "dx": _dropped(state["dy"].float(), state).to(t)} if train else {"y": y}
    if op == "low_rank_adapter":
        A, B, scale = state["A"], state["B"], state["scale"]
        xd = _dropped(x, state)
        low = xd @ A.transpose(1, 2)
        got = {"y": (state["base"].float() + scale * (low @ B.transpose(1, 2))).to(t)}
        if train:
            dy = scale * state["dy"].float()
            dlow = dy @ B
            got |= {"dx": _dropped(dlow @ A, state).to(t), "dA": dlow.transpose(1, 2) @ xd, "dB": dy.transpose(1, 2) @ low}
        return got
    if op == "layer_norm":
        y, xhat, rstd = _norm(x, state["weight"], state["bias"], state["eps"])
        got = {"y": y.to(t)}
        if train:
            dx, got["dweight"], got["dbias"] = _norm_gradients(state["dy"].float(), xhat, rstd, state["weight"])
            got["dx"] = dx.to(t)
        return got
    s = (state["residual"].float() + _dropped(x, state)).to(state["residual"].dtype)  # the sum is kept in the residual's type
    y, xhat, rstd = _norm(s.float(), state["weight"], state["bias"], state["eps"])
    got = {"y": y.to(t), "s": s}
    if train:
        dv, got["dweight"], got["dbias"] = _norm_gradients(state["dy"].float(), xhat, rstd, state["weight"])
        dv = dv + state["ds"].float()
        got |= {"dresidual": dv.to(s.dtype), "dx": _dropped(dv, state).to(t)}
    return got


# ---- the framework's operators --------------------------------------------------------------------------------------------


def _framework(state):
    from paper_2205_05632_b200 import layers
    case = state["case"]
    op, train = case["op"], case["mode"] == "train"
    leaf = (lambda k: state[k].detach().requires_grad_()) if train else (lambda k: state[k])
    x = leaf("x")
    drawn = {"p": case["p"], "seed": state["seed"], "call": state["call"]}
    if op == "dropout":
        y = layers.dropout(x, **drawn)
        return {"y": y.detach(), "dx": torch.autograd.grad(y, x, state["dy"])[0]} if train else {"y": y}
    if op == "low_rank_adapter":
        A, B = leaf("A"), leaf("B")
        y = layers.low_rank_adapter(x, state["base"], A, B, scale=state["scale"], **drawn)
        if not train:
            return {"y": y}
        dx, dA, dB = torch.autograd.grad(y, (x, A, B), state["dy"])
        return {"y": y.detach(), "dx": dx, "dA": dA, "dB": dB}
    weight, bias = leaf("weight"), leaf("bias")
    if op == "layer_norm":
        y = layers.layer_norm(x, weight, bias, eps=state["eps"])
        if not train:
            return {"y": y}
        dx, dweight, dbias = torch.autograd.grad(y, (x, weight, bias), state["dy"])
        return {"y": y.detach(), "dx": dx, "dweight": dweight, "dbias": dbias}
    residual = leaf("residual")
    y, s = layers.dropout_add_layer_norm(x, residual, weight, bias, eps=state["eps"], **drawn)
    if not train:
        return {"y": y, "s": s}
    dx, dres, dweight, dbias = torch.autograd.grad((y, s), (x, residual, weight, bias), (state["dy"], state["ds"]))
    return {"y": y.detach(), "s": s.detach(), "dx": dx, "dresidual": dres, "dweight": dweight, "dbias": dbias}


def run(state):
    if own:
        return _framework(state)
    return _plain(state)


def work(case):
    """Each input read once and each output written once; the products of the adapter, a handful of operations per element elsewhere."""
    size = {"f32": 4, "bf16": 2, "f16": 2}
    train, n, h, out, r = case["mode"] == "train", case["n"], case["h"], case["out"], case["rank"]
    m, e = n * case["rows"], size[case["dtype"]]
    if case["op"] == "dropout":
        return {"bytes": m * h * e * (4 if train else 2), "flops": m * h * (2 if train else 1)}
    if case["op"] == "low_rank_adapter":
        many = 1 if case["shared"] else n
        params = 4 * r * (h + out) * (many + (n if train else 0))
        return {"bytes": m * e * (h * (2 if train else 1) + out * (3 if train else 2)) + params,
                "flops": 2 * m * r * (h + out) * (3 if train else 1)}
    tensors = e * (4 if train else 2)
    if case["op"] == "dropout_add_layer_norm":
        tensors += size[case["residual"]] * (4 if train else 2)
    return {"bytes": m * h * tensors + 8 * h * (1 + (n if train else 0)), "flops": m * h * (20 if train else 8)}


def exact(case, seed):
    """The same from the definitions in 64 bits; gradients by differentiating the forward pass, the mask in numpy."""
    s = prepare(case, seed)
    n, rows, h, p = case["n"], case["rows"], case["h"], case["p"]
    train = case["mode"] == "train"
    dev = s["x"].device
    factor = torch.ones((), dtype=torch.float64, device=dev)
    cut = int(p * 65536 + 0.5)
    if cut:
        g = -(-h // 8)
        word = np.uint64
        low = word(0xFFFFFFFF)
        c = [np.broadcast_to(a, (n, rows, g)).astype(np.uint64) for a in
             (np.arange(g)[None, None, :], np.arange(rows)[None, :, None], np.arange(n)[:, None, None], np.full((1, 1, 1), s["call"]))]
        k0, k1 = s["seed"] % (1 << 32), s["seed"] // (1 << 32)
        for _ in range(10):
            first, second = c[0] * word(0xD2511F53), c[2] * word(0xCD9E8D57)
            c = [(second >> word(32)) ^ c[1] ^ word(k0), second & low, (first >> word(32)) ^ c[3] ^ word(k1), first & low]
            k0, k1 = (k0 + 0x9E3779B9) % (1 << 32), (k1 + 0xBB67AE85) % (1 << 32)
        bits = np.empty((n, rows, g, 8), dtype=np.uint16)
        for w in range(4):
            bits[..., 2 * w] = c[w] & word(0xFFFF)
            bits[..., 2 * w + 1] = c[w] >> word(16)
        kept = torch.from_numpy((bits >= cut) if cut < 65536 else np.zeros_like(bits, dtype=bool)).to(dev)
        factor = kept.reshape(n, rows, 8 * g)[..., :h].double() * (65536 / (65536 - cut) if cut < 65536 else 0.0)
    names = [k for k in ("x", "residual", "weight", "bias", "A", "B") if k in s]
    with torch.enable_grad():
        v = {k: s[k].double().contiguous().requires_grad_(train) for k in names}
        outputs = {}
        if case["op"] == "low_rank_adapter":
            mid = torch.einsum("nji,nri->njr", v["x"] * factor, v["A"])
            outputs["y"] = s["base"].double() + s["scale"] * torch.einsum("njr,nor->njo", mid, v["B"])
        elif case["op"] == "dropout":
            outputs["y"] = v["x"] * factor
        else:
            z = v["x"]
            if case["op"] == "dropout_add_layer_norm":
                z = v["residual"] + v["x"] * factor
                with torch.no_grad():
                    off = z.to(s["residual"].dtype).double() - z  # the sum is kept in the residual's type
                z = z + off
                outputs["s"] = z
            centred = z - z.sum(-1, keepdim=True) / h
            var = (centred * centred).sum(-1, keepdim=True) / h
            outputs["y"] = centred * (var + s["eps"]).rsqrt() * v["weight"].unsqueeze(1) + v["bias"].unsqueeze(1)
        got = {k: o.detach() for k, o in outputs.items()}
        if train:
            seeds = [s["dy"].double()] + ([s["ds"].double()] if "s" in outputs else [])
            wanted = [outputs["y"]] + ([outputs["s"]] if "s" in outputs else [])
            grads = torch.autograd.grad(wanted, [v[k] for k in names], seeds)
            got.update({"d" + k: q for k, q in zip(names, grads)})
    return got
