"""How much of the fp32 operands the adapters use. Inputs with a single number other than 0 in a row or column make every result one
product of two numbers with full significands, so an operand that lost a part of its bits shows, whatever the sizes of the sums
elsewhere.

Tolerances, in units of E = 2^-24 of the product. An fp32 number is the sum of its three bf16 planes exactly, and products of planes
are exact, so dt, t and what multiplies a one are exact. Left out are the products of planes i + j > 2: at most 8 where planes are cut
(2^-21), and 1 where they are rounded: with a in [1, 2) plane 1 is at most 2^-8 and plane 2 2^-17, so (1, 2) and (2, 1) are 2^-24
together, and 0.89 is the largest that 4 million pairs give. A sum of planes' products takes the small ones first: the last addition may
cut 2 (a unit in the last place), those before it 2^-6 of that each; fp32 additions and the scale, which is 1, round by 1 at most."""
import pytest
import torch

import operators64 as R
from paper_2205_05632_b200.layers import low_rank_adapter

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def full(g, *shape):
    """Numbers with 24 random bits, of either sign and of sizes from 2^-4 to 2^4."""
    device = g.device
    bits = torch.randint(1 << 23, 1 << 24, shape, generator=g, device=device, dtype=torch.int32).float()
    power = torch.randint(-27, -19, shape, generator=g, device=device, dtype=torch.int32)
    sign = 1.0 - 2.0 * torch.randint(0, 2, shape, generator=g, device=device, dtype=torch.int32).float()
    return torch.ldexp(bits * sign, power)


def ones_of_rows(n, rows, h, dtype, device):
    """[n, rows, h] with a one in every row, and the column of it [n, rows]."""
    at = (7 * torch.arange(rows, device=device)[None] + torch.arange(n, device=device)[:, None]) % h
    return torch.zeros(n, rows, h, dtype=dtype, device=device).scatter_(2, at[..., None], 1.0), at


def one_of_columns(g, n, rows, h, dtype, numbers=full):
    """[n, rows, h] with one number in every column, the row of it [n, h], and the numbers [n, h]."""
    at = (11 * torch.arange(h, device=g.device)[None] + torch.arange(n, device=g.device)[:, None]) % rows
    v = numbers(g, n, h).to(dtype)
    return torch.zeros(n, rows, h, dtype=dtype, device=g.device).scatter_(1, at[:, None], v[:, None]), at, v


def check(got, want, units, what):
    """Between the roundings of what is `units` E below and above."""
    tol = units * R.E * want.abs()
    lo, hi = (want - tol).to(got.dtype), (want + tol).to(got.dtype)
    bad = ~((got.cpu() >= lo) & (got.cpu() <= hi))
    assert not bad.any(), "%s: %d of %d, first at %s" % (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist())


# rows: the kernels for a few rows, mma.sync, tcgen05 (bfloat16); ranks: every form of them
SIZES = [(rows, rank) for rows in (3, 40, 200) for rank in (1, 8, 16, 24, 32, 40, 64, 100, 130)]


def pick(t, at):
    """t [n, a, b] at [n, rows] of the middle axis: [n, rows, b]."""
    return t.gather(1, at[..., None].expand(*at.shape, t.shape[-1]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,rank", SIZES)
def test_results_use_the_operands_in_full(rows, rank, dtype):
    n, h, out = 2, 136, 264
    g = torch.Generator(device="cuda").manual_seed(1)
    # y: t is a column of A, and a row of B has one number
    x, at = ones_of_rows(n, rows, h, dtype, g.device)
    a = full(g, n, rank, h)
    which = (5 * torch.arange(out, device=g.device)[None] + torch.arange(n, device=g.device)[:, None]) % rank
    b = torch.zeros(n, out, rank, device=g.device).scatter_(2, which[..., None], full(g, n, out, 1))
    want = pick(R.d(a).transpose(1, 2), at.cpu()) @ R.d(b).transpose(1, 2)  # (products with zeros: exact)
    check(low_rank_adapter(x, None, a, b), want, 12, "y")
    # dx: dt is a row of B, and a column of A has one number
    dy, at = ones_of_rows(n, rows, out, dtype, g.device)
    b = full(g, n, out, rank)
    which = (5 * torch.arange(h, device=g.device)[None] + torch.arange(n, device=g.device)[:, None]) % rank
    a = torch.zeros(n, rank, h, device=g.device).scatter_(1, which[:, None], full(g, n, 1, h))
    want = pick(R.d(b), at.cpu()) @ R.d(a)
    x = torch.zeros(n, rows, h, dtype=dtype, device=g.device, requires_grad=True)
    check(torch.autograd.grad(low_rank_adapter(x, None, a, b), x, dy)[0], want, 12, "dx")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,rank", SIZES)
def test_gradients_of_the_factors_use_t_and_dt_in_full(rows, rank, dtype):
    """The activation's planes are all of it here (one, or two), so nothing is left out: the cut of the last addition and two roundings."""
    n, h, out = 2, 136, 264
    g = torch.Generator(device="cuda").manual_seed(2)
    a, b = full(g, n, rank, h).requires_grad_(), full(g, n, out, rank).requires_grad_()
    x, at = ones_of_rows(n, rows, h, dtype, g.device)
    dy, row, v = one_of_columns(g, n, rows, out, dtype)
    t = pick(R.d(a).transpose(1, 2), at.cpu())
    db, = torch.autograd.grad(low_rank_adapter(x, None, a, b), b, dy)
    check(db, pick(t, row.cpu()) * R.d(v)[..., None], 5, "dB")
    dy, at = ones_of_rows(n, rows, out, dtype, g.device)
    x, row, v = one_of_columns(g, n, rows, h, dtype)
    dt = pick(R.d(b), at.cpu())
    da, = torch.autograd.grad(low_rank_adapter(x, None, a, b), a, dy)
    check(da, (pick(dt, row.cpu()) * R.d(v)[..., None]).transpose(1, 2), 5, "dA")


def hard(g, *shape):
    """full(), but of every two numbers one with the significand 1 + 2^-7 - 2^-23, whose planes leave most when they are cut."""
    v = full(g, *shape)
    at = torch.arange(v.numel(), device=g.device).reshape(shape) % 2 == 0
    return torch.where(at, torch.ldexp(torch.full_like(v, float(0x80ffff)), torch.frexp(v)[1] - 24) * v.sign(), v)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,rank", SIZES)
def test_planes_leave_out_no_more_than_fp32_arithmetic(rows, rank):
    """Products of two fp32 numbers, both with all of their planes. Left out 1, the last addition 2 or an fp32 one, before it 2^-5."""
    n, h, out = 2, 136, 264
    g = torch.Generator(device="cuda").manual_seed(4)
    units = 3.1
    # t: x has one number in a row, and B passes t on
    x, at = ones_of_rows(n, rows, h, F32, g.device)
    v = hard(g, n, rows, 1)
    a = hard(g, n, rank, h)
    which = (5 * torch.arange(out, device=g.device)[None] + torch.arange(n, device=g.device)[:, None]) % rank
    b = torch.zeros(n, out, rank, device=g.device).scatter_(2, which[..., None], 1.0)
    t = pick(R.d(a).transpose(1, 2), at.cpu()) * R.d(v)
    check(low_rank_adapter(x * v, None, a, b), t.gather(2, which.cpu()[:, None].expand(n, rows, out)), units, "t")
    # y, in all types: t is a column of A
    b = torch.zeros(n, out, rank, device=g.device).scatter_(2, which[..., None], hard(g, n, out, 1))
    want = pick(R.d(a).transpose(1, 2), at.cpu()) @ R.d(b).transpose(1, 2)
    for dtype in (F32, BF16, F16):
        check(low_rank_adapter(x.to(dtype), None, a, b), want, units, "y")
    # dB, dA
    a, b = a.requires_grad_(), hard(g, n, out, rank).requires_grad_()
    dy, row, v = one_of_columns(g, n, rows, out, F32, hard)
    t = pick(R.d(a).transpose(1, 2), at.cpu())
    db, = torch.autograd.grad(low_rank_adapter(x, None, a, b), b, dy)
    check(db, pick(t, row.cpu()) * R.d(v)[..., None], units, "dB")
    dy, at = ones_of_rows(n, rows, out, F32, g.device)
    x, row, v = one_of_columns(g, n, rows, h, F32, hard)
    dt = pick(R.d(b), at.cpu())
    da, = torch.autograd.grad(low_rank_adapter(x, None, a, b), a, dy)
    check(da, (pick(dt, row.cpu()) * R.d(v)[..., None]).transpose(1, 2), units, "dA")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows", [(F32, 3), (F32, 40), (F16, 40), (BF16, 40), (BF16, 200)])
def test_the_largest_numbers_and_infinities(dtype, rows):
    """Numbers that a rounding to eight bits would take beyond the largest stay finite; an infinity in a factor reaches what it should."""
    g = torch.Generator(device="cuda").manual_seed(5)
    h, out, rank = 64, 72, 8
    x, at = ones_of_rows(1, rows, h, dtype, g.device)
    big = torch.finfo(F32).max
    a, b = torch.zeros(1, rank, h, device=g.device), torch.zeros(1, out, rank, device=g.device)
    a[0, 0], a[0, 0, ::2] = big, -big
    b[0, :, 0] = 2.0 ** -126
    want = R.d(a)[0, 0][at.cpu()][..., None] * 2.0 ** -126
    check(low_rank_adapter(x, None, a, b), want.expand(1, rows, out), 3.1, "largest")
    b[0, 5, 2] = float("-inf")  # of one column of y
    a[0, 2] = 1.0
    y = low_rank_adapter(x, None, a, b)
    others = torch.arange(out, device=g.device) != 5
    assert not torch.isfinite(y[0, :, 5]).any() and torch.isfinite(y[0][:, others]).all()
    b[0, 5, 2] = 0.0
    x[0, 1] *= float("inf")  # of one row; its zeros become NaN
    y = low_rank_adapter(x, None, a, b)
    others = torch.arange(rows, device=g.device) != 1
    assert not torch.isfinite(y[0, 1]).any() and torch.isfinite(y[0, others]).all()
    x[0, 1] = 0.0
    x[0, 1, 4] = float("inf")
    assert not torch.isfinite(low_rank_adapter(x, None, a, b)[0, 1]).any()
    a[0, 1, 3] = float("inf")  # of a column of A: every row has it, times 0 or not
    assert not torch.isfinite(low_rank_adapter(x, None, a, b)).any()


def planes(v):
    """The three planes of fp32 numbers, cut."""
    out, rest = [], v.numpy().copy()
    for _ in range(3):
        high = (rest.view("uint32") & 0xffff0000).view("float32")
        out.append(torch.from_numpy(high).double())
        rest = rest - high
    return out


def test_a_plane_that_is_left_out_would_show():
    """The same checks on sums of products that lack one plane of one operand, which fail."""
    g = torch.Generator().manual_seed(3)
    t, f, x = full(g, 20000), full(g, 20000), full(g, 20000).to(BF16).double()
    pt, pf = planes(t), planes(f)
    assert torch.equal(sum(pt), t.double()) and torch.equal(sum(pf), f.double())
    check(sum(pt[i] * pf[j] for i in range(3) for j in range(3 - i)).float(), t.double() * f.double(), 12, "all of them")
    check((sum(pt) * x).float(), t.double() * x, 5, "all of them")
    for gone in range(3):
        with pytest.raises(AssertionError):
            check((sum(pt[i] for i in range(3) if i != gone) * x).float(), t.double() * x, 5, "dA, dB")
        for type_ in (F32, BF16, F16):
            with pytest.raises(AssertionError):
                check(sum(pt[i] * pf[j] for i in range(3) for j in range(3 - i) if i != gone).to(type_), t.double() * f.double(), 12, "y, dx")
