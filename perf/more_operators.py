"""Performance cases of the operators around a model's blocks and at the two ends of its backward pass, for the n workers'
micro-batches in one batch: activations [n, rows, h] with the worker in front, each worker's gradients kept apart where the
parameter is a leaf with a row for every worker.

    linear_cross_entropy    the head: logits z = x W^T over a vocabulary, softmax cross entropy with the targets, the mean over
                            each worker's counted targets; gradients of x and W. The logits are never stored as a whole.
    rms_norm                x / sqrt(mean(x^2) + eps) * weight
    gated_add_rms_norm      s = residual_scale * residual + gate * rms_norm(x, weight), the norm behind a block with its gate and
                            the residual's scale, and rms_norm(s, next_weight), the norm before the next block
    collect_gradients       many tensors' gradients, a worker's in each row, gathered as the rows of G [n, d]; every worker's
                            global norm, and rows above max_norm scaled by max_norm / (norm + 1e-6)

"infer" passes run forward, "train" passes forward and backward.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IGNORED = -100
EPS = 1e-6


def head(name, n, rows, h, vocab, dtype="bf16", wtype="", weight="shared", wanted="", ignored=0.0):
    """weight: "shared" [vocab, h], its gradient summed over the workers; "apart": the same for all, seen by each, gradients apart;
    "own": one per worker. wanted: the gradients, "", "x" (a head that is not trained) or "xw"."""
    c = {"op": "head", "n": n, "rows": rows, "h": h, "vocab": vocab, "dtype": dtype, "wtype": wtype or dtype, "weight": weight,
         "wanted": wanted, "ignored": ignored}
    return {"name": name, **c} if name else c


def norm(name, op, mode, n, rows, h, dtype="bf16", residual=""):
    c = {"op": op, "mode": mode, "n": n, "rows": rows, "h": h, "dtype": dtype, "residual": residual or dtype}
    return {"name": name, **c} if name else c


def collect(name, n, blocks, width, dtype="f32", share=0.5):
    """Gradients of `blocks` blocks of a model (_shapes) of n workers, a share of which is over max_norm."""
    c = {"op": "collect", "n": n, "blocks": blocks, "width": width, "dtype": dtype, "share": share}
    return {"name": name, **c} if name else c


def listed():
    return [
        # scoring one token while answering: latency, and the weight is read once
        head("head one token", 1, 1, 4096, 32000),
        # fine-tuning under a head that is not trained, a vocabulary of no round size, padding in the batch
        head("head bf16 n=8 frozen", 8, 512, 2048, 50257, wanted="x", ignored=0.2),
        # a small full-precision model, ragged micro-batches, every worker's gradient of the head apart
        head("head f32 n=4", 4, 100, 512, 8000, "f32", weight="apart", wanted="xw"),
        # mixed precision over full-precision parameters, as the optimizer keeps them, gradients apart
        head("head bf16/f32 n=8", 8, 256, 1024, 32000, "bf16", "f32", "apart", "xw", 0.1),
        # a large head trained for all workers together
        head("head bf16 n=8 largest", 8, 1024, 4096, 100000, wanted="xw", ignored=0.1),
        # one token of each of 32 requests
        norm("norm 32 tokens h=4096", "rms_norm", "infer", 32, 1, 4096),
        # micro-batches of eight workers
        norm("norm bf16 n=8 h=2048", "rms_norm", "train", 8, 2048, 2048),
        # one token while answering, a block's end
        norm("block norms one token h=4096", "gated", "infer", 1, 1, 4096),
        # a block's end in half precision, the residual stream in full precision, an odd width
        norm("block norms f16/f32 n=3 h=1001", "gated", "train", 3, 777, 1001, "f16", "f32"),
        # eight workers with long micro-batches
        norm("block norms bf16 n=8 h=4096", "gated", "train", 8, 2048, 4096),
        # adapters and norms of a small model: latency
        collect("collect n=4 small", 4, 6, 96),
        # a model of 11 million parameters, half the workers are clipped
        collect("collect n=16", 16, 12, 276),
    ]


def _spread(rng, low, high):
    """A size between the two, evenly over its logarithm; as a rule, but not always, a multiple of 8."""
    v = int(math.exp(rng.uniform(math.log(low), math.log(high + 1.0))))
    return v if v < 16 or rng.random() < 0.4 else v // 8 * 8


def draw(rng: random.Random):
    op = rng.choice(["head", "head", "rms_norm", "gated", "collect"])
    if op == "head":
        dtype, wtype = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f16", "f16"), ("f16", "f32")])
        n, rows, h, vocab = _spread(rng, 1, 16), _spread(rng, 1, 2048), _spread(rng, 64, 4096), _spread(rng, 1000, 131072)
        weight, wanted = rng.choice(["shared", "shared", "apart", "own"]), rng.choice(["", "x", "xw", "xw"])
        while n * rows * vocab > 8192 * 100000 or n * rows * h * vocab > (3 << 40 if dtype == wtype != "f32" else 1 << 38):
            rows = rows // 2 + rng.randrange(2) if rows > 2 else 1
            n, vocab = (n, vocab) if rows > 1 else (max(1, n // 2), max(1000, vocab // 2))
        while vocab * h * (n if weight == "own" or (weight, wanted) == ("apart", "xw") else 1) > 1 << 29:
            vocab = vocab // 2 + rng.randrange(2)
        return head("", n, rows, h, vocab, dtype, wtype, weight, wanted, rng.choice([0.0, 0.1, 0.5]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    n = _spread(rng, 1, 32)
    if op == "collect":
        blocks, width = rng.randint(1, 24), _spread(rng, 8, 512)
        while n * blocks * 12 * width * width > 160 << 20:
            width, blocks = width // 2 + rng.randrange(8), max(1, blocks - 1)
        return collect("", n, blocks, width, dtype, rng.choice([0.0, 0.5, 1.0]))
    rows, h = _spread(rng, 1, 8192), _spread(rng, 8, 16384)
    residual = rng.choice([dtype, "f32"]) if op == "gated" else dtype
    while n * rows * h > (1 << 25 if "f32" in (dtype, residual) else 1 << 26):
        rows = rows // 2 + rng.randrange(2) if rows > 2 else 1
        n = n if rows > 1 else max(1, n // 2)
    return norm("", op, "train" if rng.random() < 0.7 else "infer", n, rows, h, dtype, residual)


def _shapes(blocks, width):
    """Parameters of a model of `blocks` transformer blocks, without its embedding: norms, projections, biases."""
    block = [(width,), (3 * width, width), (3 * width,), (width, width), (width,), (width,), (4 * width, width), (4 * width,),
             (width, 4 * width), (width,)]
    return block * blocks + [(width,), (7, width), (7,)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t, n = TYPES[case["dtype"]], case["n"]

    def normal(*shape, sigma=1.0, dtype=torch.float32):
        return (sigma * torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)).to(dtype)

    s = {"case": case}
    if case["op"] == "collect":
        # tensors' gradients of different sizes, workers' of different norms
        shapes = _shapes(case["blocks"], case["width"])
        d = sum(math.prod(shape) for shape in shapes)
        far = torch.rand(n, generator=gen, device="cuda") < case["share"]
        size = torch.where(far, 2.0, 0.25) * (1.0 + 0.5 * torch.rand(n, generator=gen, device="cuda")) / d ** 0.5
        s["grads"] = [normal(n, *shape, dtype=t).mul_(size.to(t).view(n, *[1] * len(shape))) for shape in shapes]
        s["out"], s["max_norm"] = torch.empty(n, d, device="cuda"), 1.0
        return s
    rows, h = case["rows"], case["h"]
    if case["op"] == "head":
        # a head whose logits have a deviation of about 2.5, hidden states that lean to their targets' rows, frequent targets and rare ones
        vocab, w = case["vocab"], TYPES[case["wtype"]]
        many = (n,) if case["weight"] == "own" else ()
        s["weight"] = normal(*many, vocab, h, sigma=2.5 * h ** -0.5, dtype=w)
        s["target"] = (vocab * torch.rand(n, rows, generator=gen, device="cuda").pow(3)).long().clamp_(0, vocab - 1)
        toward = torch.stack([s["weight"][i][s["target"][i]] for i in range(n)]) if many else s["weight"][s["target"]]
        s["x"] = (normal(n, rows, h) + toward.float()).to(t)
        s["target"] = torch.where(torch.rand(n, rows, generator=gen, device="cuda") < case["ignored"], IGNORED, s["target"])
        if case["weight"] == "apart":
            s["weight"] = s["weight"].expand(n, vocab, h)
        s["dloss"] = torch.full((n,), 4096.0 if case["dtype"] == "f16" else 1.0, device="cuda")  # half precision: with a loss scale
        return s
    # activations: channels of different sizes
    s["x"] = (normal(n, rows, h) * (0.5 + normal(h).abs())).to(t)
    s["weight"] = (1.0 + 0.2 * normal(h)).expand(n, h)
    if case["op"] == "gated":
        s["residual"] = normal(n, rows, h, sigma=2.0, dtype=TYPES[case["residual"]])
        s["gate"], s["next_weight"], s["scale"] = (0.5 + 0.2 * normal(h)).expand(n, h), (1.0 + 0.2 * normal(h)).expand(n, h), 0.9
    if case["mode"] == "train":
        s["dy"] = normal(n, rows, h, sigma=0.02, dtype=t)
        if case["op"] == "gated":
            s["ds"] = normal(n, rows, h, sigma=0.02, dtype=TYPES[case["residual"]])
    return s


# ---- the operators in their plain form ------------------------------------------------------------------------------------


def _plain_head(state):
    case, x, target = state["case"], state["x"].float(), state["target"]
    weight = state["weight"][0] if case["weight"] == "apart" else state["weight"]
    W, counted = weight.float(), target != IGNORED
    at = torch.where(counted, target, 0).unsqueeze(-1)
    z = x @ W.transpose(-1, -2)
    of_target = z.gather(-1, at).squeeze(-1)
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(-1, keepdim=True)
    row = torch.where(counted, (top + total.log()).squeeze(-1) - of_target, 0.0)
    count = counted.sum(1).clamp(min=1)
    got = {"loss": row.sum(1) / count}
    if not case["wanted"]:
        return got
    dz = e.div_(total)
    dz.scatter_add_(-1, at, torch.full_like(of_target, -1.0).unsqueeze(-1))
    dz.mul_((counted * (state["dloss"] / count)[:, None]).unsqueeze(-1))
    got["dx"] = (dz @ W).to(state["x"].dtype)
    if "w" in case["wanted"]:
        if case["weight"] == "shared":
            dW = dz.flatten(0, 1).t() @ x.flatten(0, 1)
        else:
            dW = dz.transpose(1, 2) @ x
        got["dweight"] = dW.to(weight.dtype)
    return got


def _rms(v, eps):
    return 1.0 / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)


def _rms_gradient(dy, v, r, w):
    """Of v * r * w: gradients of v and w, r being the reciprocal root of v's mean square."""
    g = dy * w[:, None]
    vhat = v * r
    return r * (g - vhat * (g * vhat).mean(-1, keepdim=True)), (dy * vhat).sum(1)


def _plain_norm(state):
    case, t = state["case"], TYPES[state["case"]["dtype"]]
    x, w = state["x"].float(), state["weight"]
    r = _rms(x, EPS)
    u = x * r * w[:, None]
    if case["op"] == "rms_norm":
        got = {"y": u.to(t)}
        if case["mode"] == "train":
            dx, got["dweight"] = _rms_gradient(state["dy"].float(), x, r, w)
            got["dx"] = dx.to(t)
        return got
    gate, alpha = state["gate"], state["scale"]
    # kept in the residual's type: formed in 64 bits, so that what lies next to a border of bfloat16 is rounded to its side of it
    wide = x.double()
    wide = wide * _rms(wide, EPS) * (gate * w.double())[:, None]
    s = wide.add_(state["residual"], alpha=alpha).to(state["residual"].dtype)
    v, w2 = s.float(), state["next_weight"]
    q = _rms(v, EPS)
    got = {"y": (v * q * w2[:, None]).to(t), "s": s}
    if case["mode"] == "train":
        dv, got["dnext"] = _rms_gradient(state["dy"].float(), v, q, w2)
        dv = dv + state["ds"].float()
        dx, got["dweight"] = _rms_gradient(dv * gate[:, None], x, r, w)
        got |= {"dgate": (dv * u).sum(1), "dresidual": (alpha * dv).to(s.dtype), "dx": dx.to(t)}
    return got


def _plain_collect(state):
    n, grads = state["case"]["n"], state["grads"]
    rows = torch.cat([g.reshape(n, -1).float() for g in grads], dim=1)
    squares = torch.stack([g.reshape(n, -1).float().square().sum(1, dtype=torch.float64) for g in grads])
    norms = squares.sum(0).sqrt()
    factor = (state["max_norm"] / (norms + 1e-6)).clamp(max=1.0).float()
    return {"G": rows * factor[:, None], "norms": norms.float()}


# ---- the framework's operators --------------------------------------------------------------------------------------------


def _framework(state):
    from paper_2205_05632_b200 import layers, optim
    case = state["case"]
    if case["op"] == "collect":
        G, norms = optim.collect_gradients(state["grads"], out=state["out"], max_norm=state["max_norm"])
        return {"G": G, "norms": norms}
    if case["op"] == "head":
        wanted = case["wanted"]
        x = state["x"].detach().requires_grad_("x" in wanted)
        weight = state["weight"].detach().requires_grad_("w" in wanted)
        loss = layers.linear_cross_entropy(x, weight, state["target"])
        if not wanted:
            return {"loss": loss}
        grads = torch.autograd.grad(loss, (x, weight) if "w" in wanted else (x,), state["dloss"])
        return {"loss": loss.detach(), **dict(zip(("dx", "dweight"), grads))}
    train = case["mode"] == "train"
    leaf = (lambda k: state[k].detach().requires_grad_()) if train else (lambda k: state[k])
    x, weight = leaf("x"), leaf("weight")
    if case["op"] == "rms_norm":
        y = layers.rms_norm(x, weight, eps=EPS)
        if not train:
            return {"y": y}
        dx, dweight = torch.autograd.grad(y, (x, weight), state["dy"])
        return {"y": y.detach(), "dx": dx, "dweight": dweight}
    residual, gate, after = leaf("residual"), leaf("gate"), leaf("next_weight")
    y, s = layers.gated_add_rms_norm(x, residual, weight, gate, after, residual_scale=state["scale"], eps=EPS)
    if not train:
        return {"y": y, "s": s}
    dx, dres, dweight, dgate, dnext = torch.autograd.grad((y, s), (x, residual, weight, gate, after), (state["dy"], state["ds"]))
    return {"y": y.detach(), "s": s.detach(), "dx": dx, "dresidual": dres, "dweight": dweight, "dgate": dgate, "dnext": dnext}


def run(state):
    if own:
        return _framework(state)
    if state["case"]["op"] == "collect":
        return _plain_collect(state)
    return _plain_head(state) if state["case"]["op"] == "head" else _plain_norm(state)


def work(case):
    """Each input read once and each output written once; the head's products (one forward, one for each gradient), a handful of
    operations an element elsewhere."""
    size = {"f32": 4, "bf16": 2, "f16": 2}
    n, e = case["n"], size[case["dtype"]]
    if case["op"] == "collect":
        d = sum(math.prod(shape) for shape in _shapes(case["blocks"], case["width"]))
        return {"bytes": n * d * (e + 4) + 4 * n, "flops": 3 * n * d}
    m, h = n * case["rows"], case["h"]
    if case["op"] == "head":
        wanted, w = case["wanted"], size[case["wtype"]] * case["vocab"] * h
        weights = w * (n if case["weight"] == "own" else 1)
        gradients = w * (1 if case["weight"] == "shared" else n) if "w" in wanted else 0
        return {"bytes": weights + gradients + m * h * e * (2 if "x" in wanted else 1) + 8 * m + 4 * n,
                "flops": 2 * m * h * case["vocab"] * (1 + len(wanted))}
    train = case["mode"] == "train"
    tensors = e * (4 if train else 2)
    if case["op"] == "gated":
        tensors += size[case["residual"]] * (4 if train else 2)
    weights = 3 if case["op"] == "gated" else 1
    return {"bytes": m * h * tensors + 4 * h * weights * (1 + (n if train else 0)), "flops": m * h * (15 if train else 5) * (2 if weights > 1 else 1)}


def exact(case, seed):
    """The same from the definitions in 64 bits; gradients by differentiating the forward pass."""
    s = prepare(case, seed)
    n = case["n"]
    if case["op"] == "collect":
        G, norms, done = torch.empty(s["out"].shape, dtype=torch.float64, device=s["out"].device), [], 0
        for g in s["grads"]:
            flat = g.reshape(n, -1)
            G[:, done:done + flat.shape[1]] = flat
            done += flat.shape[1]
        for i in range(n):
            norms.append(torch.linalg.vector_norm(G[i]))
            if float(norms[i]) + 1e-6 > s["max_norm"]:
                G[i] *= s["max_norm"] / (norms[i] + 1e-6)
        return {"G": G, "norms": torch.stack(norms)}
    if case["op"] == "head":
        wanted, losses, dx, dW = case["wanted"], [], [], []
        with torch.enable_grad():
            for i in range(n):  # a worker at a time
                W = (s["weight"] if s["weight"].dim() == 2 else s["weight"][i]).double().requires_grad_("w" in wanted)
                x = s["x"][i].double().requires_grad_("x" in wanted)
                here = (s["target"][i] != IGNORED).nonzero().flatten()
                if here.numel():
                    z = torch.einsum("jk,vk->jv", x[here], W)
                    loss = (torch.logsumexp(z, -1) - z[torch.arange(len(here), device=z.device), s["target"][i][here]]).mean()
                else:
                    loss = 0.0 * (x.sum() + W.sum())
                losses.append(loss.detach())
                if wanted:
                    g = torch.autograd.grad(loss, (x, W) if "w" in wanted else (x,), s["dloss"][i].double())
                    dx.append(g[0])
                    if "w" in wanted and case["weight"] == "shared" and dW:
                        dW[0] += g[1]
                    elif "w" in wanted:
                        dW.append(g[1])
                    del g
                z = loss = None
        got = {"loss": torch.stack(losses)}
        if wanted:
            got["dx"] = torch.stack(dx)
        if "w" in wanted:
            got["dweight"] = dW[0] if case["weight"] == "shared" else torch.stack(dW)
        return got
    train = case["mode"] == "train"
    names = [k for k in ("x", "residual", "weight", "gate", "next_weight") if k in s]
    with torch.enable_grad():
        v = {k: s[k].double().contiguous().requires_grad_(train) for k in names}

        def normed(a, w):
            return a * w.unsqueeze(1) / (torch.einsum("njc,njc->nj", a, a).unsqueeze(-1) / case["h"] + EPS).sqrt()

        out = {"y": normed(v["x"], v["weight"])}
        if case["op"] == "gated":
            total = s["scale"] * v["residual"] + v["gate"].unsqueeze(1) * out["y"]
            with torch.no_grad():
                off = total.to(s["residual"].dtype).double() - total  # the sum is kept in the residual's type
            out["s"] = total + off
            out["y"] = normed(out["s"], v["next_weight"])
        got = {k: o.detach() for k, o in out.items()}
        if train:
            keys = [k for k in ("y", "s") if k in out]
            grads = torch.autograd.grad([out[k] for k in keys], [v[k] for k in names], [s["d" + k].double() for k in keys])
            got.update({"dnext" if k == "next_weight" else "d" + k: g for k, g in zip(names, grads)})
    return got
