"""collect_gradients, clip_gradients, collect_all(max_norm) and clip() against 64 bits: places, types, boundaries, norms at both ends of the
range, what is not finite, strides, streams, graphs."""
import pytest
import torch

from paper_2205_05632_b200 import BLOCKSIGN, CompAMSError
from paper_2205_05632_b200.optim import CompAMSOptimizer, clip_gradients, collect_gradients

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PIECE = 8192
SIZES = [[1], [2, 1, 3], [PIECE - 1, PIECE, PIECE + 1, 5], [3, 2 * PIECE, 1, 3 * PIECE + 2], [7] * 320, [5] * 321 + [PIECE, 9], [40000, 1, 2, 3]]


def gradients(seed, sizes, n, kinds, phase=0):
    """Tensors [n, size], each a few elements past an allocation's start; worker i's about i + 1 times as large."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    got = []
    for k, s in enumerate(sizes):
        t = torch.randn(n * s + phase, generator=g, device="cuda")[phase:].view(n, s) * torch.arange(1, n + 1, device="cuda")[:, None]
        kind = kinds[k % len(kinds)]
        out = torch.empty(n * s + phase, dtype=kind, device="cuda")[phase:].view(n, s)
        got.append(out.copy_(t))
    return got


def expected(grads, max_norm, eps=1e-6):
    """G in 64 bits, whether a row is as it was, norms."""
    rows = torch.cat([t.reshape(t.shape[0], -1).double() for t in grads], 1)
    norms = rows.square().sum(1).sqrt()
    f = (max_norm / (norms + eps)).clamp(max=1.0)
    return rows * f[:, None], f == 1.0, norms


def close(got, want, steps, kind=F32):
    """Within so many roundings; a unit of the smallest."""
    u = torch.finfo(kind).eps / 2
    tiny = 2.0 ** -24 if kind == F16 else 2.0 ** -133 if kind == BF16 else 2.0 ** -149
    return bool(((got.double() - want).abs() <= steps * u * want.abs() + tiny).all())


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: str(len(s)) + "x" + str(max(s)))
@pytest.mark.parametrize("kinds", [(F32,), (BF16,), (F16,), (F32, F16, BF16)], ids=str)
@pytest.mark.parametrize("phase", [0, 1, 2, 3])
def test_gathered_and_clipped(sizes, kinds, phase):
    n = 5
    grads = gradients(len(sizes), sizes, n, kinds, phase)
    d = sum(sizes)
    limit = 2.5 * d ** 0.5  # the first workers are below, the last above
    want, same, norms = expected(grads, limit)
    out = torch.full((n, d + 3), float("nan"), device="cuda")
    G, got = collect_gradients(grads, out=out[:, phase:phase + d], max_norm=limit)
    # the norm is summed in binary64 but for fours of squares: 4 roundings, half of which the root leaves, and the last
    assert close(got, norms, 4)
    assert G.data_ptr() == out[:, phase:].data_ptr() and torch.isnan(out[:, :phase]).all() and torch.isnan(out[:, phase + d:]).all()
    rows = torch.cat([t.float().reshape(n, -1) for t in grads], 1)
    assert torch.equal(G[same], rows[same])
    assert close(G, want, 8)  # the factor carries the norm's error
    # in place, each tensor in its own type
    kept = [t.clone() for t in grads]
    again = clip_gradients(grads, limit)
    assert torch.equal(again, got)
    lo = 0
    for t, was in zip(grads, kept):
        assert torch.equal(t[same], was[same])
        assert close(t, want[:, lo:lo + t.shape[1]], 9 if t.dtype == F32 else 1.1, t.dtype)
        lo += t.shape[1]
    # nothing to clip: a copy
    G, got = collect_gradients(kept)
    assert torch.equal(G, rows) and close(got, norms, 4)


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e18, 1e30, 3e38])
def test_squares_that_fp32_does_not_hold(size):
    g = torch.Generator(device="cuda").manual_seed(1)
    t = size * (0.5 + 0.5 * torch.rand(3, 5000, generator=g, device="cuda"))
    norms = t.double().square().sum(1).sqrt()
    _, got = collect_gradients([t])
    inside = norms < torch.finfo(F32).max
    assert close(got[inside], norms[inside], 4) and torch.isinf(got[~inside]).all()
    limit = 0.25 * size
    G, _ = collect_gradients([t], max_norm=limit, eps=0.0)
    assert close(G, t.double() * (limit / norms)[:, None], 8)


def test_values_that_are_not_finite():
    t = torch.ones(4, 9000, device="cuda")
    t[1, 8999], t[2, 0], t[3, 17] = float("inf"), float("nan"), -float("inf")
    kept = t.clone()
    G, norms = collect_gradients([t], max_norm=1e9)
    assert torch.isinf(norms[1]) and torch.isnan(norms[2]) and torch.isinf(norms[3])
    assert torch.equal(G[0], t[0]) and torch.isnan(G[2]).all()
    assert torch.isnan(G[1, 8999]) and not G[1, :8999].any()  # a factor of 0
    clip_gradients([t], 1e9)
    assert torch.equal(t.isnan(), G.isnan()) and torch.equal(t.nan_to_num(), G.nan_to_num())
    G, _ = collect_gradients([kept])  # not clipped: as they were
    assert torch.equal(G.view(torch.int32), kept.view(torch.int32))
    zero = torch.zeros(2, 100, device="cuda")
    G, norms = collect_gradients([zero], max_norm=1.0)
    assert not G.any() and not norms.any()
    G, _ = collect_gradients([torch.ones(2, 100, device="cuda")], max_norm=0.0)
    assert not G.any()


def test_layouts():
    g = torch.Generator(device="cuda").manual_seed(2)
    base = torch.randn(4, 30, 50, generator=g, device="cuda")
    grads = [base.transpose(1, 2), base[:, :, 3:], base[:, 0], base[:, :1, :1].expand(4, 7, 9), torch.zeros(4, 0, 5, device="cuda")]
    G, norms = collect_gradients(grads, max_norm=10.0)
    want, _, exact = expected(grads, 10.0)
    assert close(G, want, 8) and close(norms, exact, 4)
    wide = torch.randn(4, 100, generator=g, device="cuda")
    part = wide[:, 5:77]  # workers further apart than their elements
    kept = wide.clone()
    want, _, exact = expected([part], 1.0)
    assert close(clip_gradients([part], 1.0), exact, 4) and close(part, want, 9)
    assert torch.equal(wide[:, :5], kept[:, :5]) and torch.equal(wide[:, 77:], kept[:, 77:])
    for bad in (base.transpose(1, 2), base[:, :, 3:], base[:1].expand(4, 30, 50), torch.zeros(3, device="cuda", requires_grad=True)):
        with pytest.raises(CompAMSError):
            clip_gradients([bad], 1.0)
    flat = torch.randn(9, generator=g, device="cuda")  # a scalar parameter: one element a worker
    assert close(collect_gradients(flat)[1], flat.double().abs(), 4)


def test_autograd_knows_what_was_written():
    x = torch.randn(2, 10, device="cuda", requires_grad=True)
    y = x * 3.0
    z = (y * y).sum()
    clip_gradients(y, 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


@pytest.mark.parametrize("sizes", [[1], [7, 3, 40000, 2], [PIECE + 3] * 5, [3] * 400])
@pytest.mark.parametrize("max_norm", [None, 5.0])
def test_the_optimizer_collects_and_clips(sizes, max_norm):
    n = 3
    params = [torch.nn.Parameter(torch.zeros(s, device="cuda")) for s in sizes]
    opt = CompAMSOptimizer(params, n, BLOCKSIGN, whole_vector=True)
    opt.G.fill_(float("nan"))
    grads = gradients(9, sizes, n, (F32,), 1)
    for k, (leaf, g) in enumerate(zip(opt.worker_parameters(), grads)):
        leaf.grad = None if k % 3 == 1 else g.clone()
    want, same, norms = expected([torch.zeros_like(g) if k % 3 == 1 else g for k, g in enumerate(grads)], max_norm or float("inf"))
    got = opt.collect_all(max_norm) if max_norm else opt.collect_all()
    assert close(opt.G, want, 8) and all(leaf.grad is None for leaf in opt.worker_parameters())
    assert got is None if max_norm is None else close(got, norms, 4)
    if max_norm is None:
        assert torch.equal(opt.G.double(), want)
        assert close(opt.clip(5.0), norms, 4)
        assert close(opt.G, expected([want], 5.0)[0], 8)
    opt.step()
    opt.close()


def test_long_rows():
    n, d = 3, (1 << 27) + 5
    g = torch.Generator(device="cuda").manual_seed(3)
    t = torch.randn(n, d, generator=g, device="cuda")
    norms = torch.stack([r.double().square().sum().sqrt() for r in t])
    G, got = collect_gradients([t], max_norm=1000.0)
    assert close(got, norms, 4)
    for i in range(n):
        for k in (0, d // 2, d - 5000):
            assert close(G[i, k:k + 5000], t[i, k:k + 5000].double() * (1000.0 / (norms[i] + 1e-6)), 8)
    again = collect_gradients([t], out=G, max_norm=1000.0)[1]
    assert torch.equal(again, got)


def test_offsets_beyond_32_bits():
    n, d = 2, (1 << 31) // 2 + 777  # worker 1 starts beyond 2^30 elements, ends beyond 2^31
    t = torch.zeros(n, d, dtype=BF16, device="cuda")
    t[1, -3:], t[0, 5] = 3.0, 4.0
    G, norms = collect_gradients([t], max_norm=1.0, eps=0.0)
    assert float(norms[0]) == 4.0 and abs(float(norms[1]) - 27 ** 0.5) < 1e-6
    assert float(G[0, 5]) == 1.0 and abs(float(G[1, -1]) - 3 / 27 ** 0.5) < 1e-7 and not G[1, :-3].any()
    del G
    clip_gradients([t], 1.0, eps=0.0)
    assert float(t[0, 5]) == 1.0 and abs(float(t[1, -1]) - 3 / 27 ** 0.5) < 2.0 ** -9


def test_captured_and_on_two_streams():
    grads = gradients(4, [300, 70000, 5], 4, (F32, BF16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = torch.zeros(4, 70305, device="cuda")
        collect_gradients(grads, out, 10.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _, norms = collect_gradients(grads, out, 10.0)
    torch.cuda.current_stream().wait_stream(side)
    for t in grads:
        t.mul_(-2.0)
    graph.replay()
    torch.cuda.synchronize()
    want, exact = collect_gradients(grads, max_norm=10.0)
    assert torch.equal(out, want) and torch.equal(norms, exact)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    many = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                many.append(collect_gradients(grads, max_norm=10.0))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) and torch.equal(b, exact) for a, b in many)


def test_refusals():
    t = torch.zeros(2, 8, device="cuda")
    for bad in ([], [None], [t, torch.zeros(3, 8, device="cuda")], [t, t.cpu()], [t.double()], [t.cpu()], [torch.zeros((), device="cuda")], [t[:0]]):
        with pytest.raises(CompAMSError):
            collect_gradients(bad)
        with pytest.raises(CompAMSError):
            clip_gradients(bad, 1.0)
    for out in (torch.zeros(2, 7, device="cuda"), torch.zeros(2, 8), torch.zeros(2, 8, dtype=BF16, device="cuda"), torch.zeros(8, 2, device="cuda").t(),
                torch.zeros(1, 8, device="cuda").expand(2, 8), 3):
        with pytest.raises(CompAMSError):
            collect_gradients([t], out=out)
    for limit in (-1.0, float("nan")):
        with pytest.raises(CompAMSError):
            collect_gradients([t], max_norm=limit)
        with pytest.raises(CompAMSError):
            clip_gradients([t], limit)
    with pytest.raises(CompAMSError):
        clip_gradients([t], 1.0, eps=-1.0)


def test_tensors_that_overlap():
    wide = torch.randn(3, 40, device="cuda")
    want = wide.double()
    norms = want.norm(dim=1)
    for bad in ([wide, wide], [wide[:, :21], wide[:, 20:]], [wide, wide[:1].expand(3, 40)[:, :0], wide]):
        with pytest.raises(CompAMSError):
            clip_gradients(bad, 1.0)
    for bad in ([wide], [wide[1, :3], wide.new_zeros(3, 39)], (wide.new_zeros(3, 39), wide.view(-1)[117:])):
        with pytest.raises(CompAMSError):
            collect_gradients(bad, out=wide)
    assert torch.equal(wide.double(), want)
    G, all_norms = collect_gradients([wide, wide])  # read only: it may stand there twice
    assert torch.equal(G, torch.cat([wide, wide], 1)) and close(all_norms, norms * 2 ** 0.5, 4)
    got = clip_gradients([wide[:, :21], wide[:, 21:]], 1.0, eps=0.0)  # beside one another
    assert close(got, norms, 4) and close(wide, want * (1.0 / norms).clamp(max=1.0)[:, None], 9)
