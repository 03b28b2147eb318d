"""What long depths may cost the cross entropy's gradients: nothing that grows with the depth.

The tensor cores cut off what an accumulator's last bit cannot hold, so an accumulation of one-signed terms shrinks with every
step of 16.  u = 2^-24; h half a step of the inputs' type relative to the value (bfloat16 2^-8, float16 2^-11)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# An accumulation that is cut into pieces of 1 024: 64 steps, each of which cuts off less than 2 u of it
PIECE = 64 * 2 * U32


@pytest.fixture(scope="module")
def ops():
    from paper_2605_17879_b200 import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,far", [(512, 40.0), (1024, 300.0), (1032, 40.0), (2048, 40.0), (2048, 300.0), (4096, 40.0), (4096, 300.0)])
def test_a_certain_target_is_left_alone(ops, dtype, d, far):
    """Rows whose target has all the probability (the others lie `far` below): G at the target is 0, and dx with it.  Every
    product of the target's logit is positive."""
    n, v = 192, 300
    g = gen(d)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") * (0.5 / math.sqrt(d))).to(dtype)
    t = torch.arange(n, device="cuda")
    w[:n] = (x.double() * (far / d)).to(dtype)
    z = x.double() @ w.double().T
    at = z.gather(1, t[:, None])[:, 0]
    gap = at - z.scatter(1, t[:, None], -math.inf).amax(1)
    assert float(gap.min()) > 17 + math.log(v)             # (others: below 2^-24 in all)
    one = torch.ones(1, device="cuda")
    out = ops.linear_xent(x, w, t)
    dx = ops.linear_xent_grad(x, w, t, out["lse"], one)["dx"].double()
    wt = w[:n].double()
    G = (dx * wt).sum(1) / (wt * wt).sum(1)                # G at the target, as dx holds it
    # The log sum is the target's logit but for the rounding of an exponent (u of it, twice), of the sum (u of it), an
    # exponential and a logarithm (2^-22 each); the other entries' share; the rounding of G and of dx is relative.
    others = math.exp(-float(gap.min())) * v * 4           # (their rows of w are no longer than the target's by a factor of 4)
    tol = (3 * U32 * at.abs() + 2.0 ** -21) * (1 + 3 * HALF[dtype]) + others
    # a float16 dx also rounds to 2^-25 absolutely, in a direction of its own per element
    tol = tol + (2.0 ** -25 * math.sqrt(d) / wt.norm(dim=1) if dtype == torch.float16 else 0.0)
    assert (G.abs() <= tol).all(), (float((G.abs() / tol).max()), float(G.mean()))


@pytest.mark.parametrize("n", [100, 500])
def test_rows_that_move_keep_their_logits(ops, n):
    """With rows ignored the backward pass finds a row elsewhere in its tile than the forward pass did (100 rows, taken as they
    are there), or both find it elsewhere than without: the same bits."""
    d, v = 2056, 700
    g = gen(n)
    x = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * (2 / math.sqrt(d))).bfloat16()
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    some = torch.where(torch.arange(n, device="cuda") % 3 == 0, -100, t)
    one = torch.ones(1, device="cuda")
    full, part = ops.linear_xent(x, w, t), ops.linear_xent(x, w, some)
    keep = some >= 0
    assert torch.equal(full["loss"][keep], part["loss"][keep]) and torch.equal(full["lse"][keep], part["lse"][keep])
    # (dx takes all of the row's G, and its split goes by the number of tiles, which is the same)
    a, b = ops.linear_xent_grad(x, w, t, full["lse"], one)["dx"], ops.linear_xent_grad(x, w, some, part["lse"], one)["dx"]
    if n == 100:
        assert torch.equal(a[keep], b[keep])
    else:                                                  # two row tiles against three: another grouping of float32 sums
        assert ((a[keep].double() - b[keep].double()).abs() <= 2 * HALF[torch.bfloat16] * a[keep].double().abs() + 2.0 ** -20).all()


def one_signed(seed, n, d, v, dtype, sx, sw):
    """x of either sign and w positive, small logits; every target is entry 0, whose row of w is zero: all terms of dx are
    positive."""
    g = gen(seed)
    sign = torch.randint(0, 2, (n, d), generator=g, device="cuda") * 2 - 1
    x = ((torch.rand(n, d, generator=g, device="cuda") + 0.5) * sign * sx).to(dtype)
    w = ((torch.rand(v, d, generator=g, device="cuda") + 0.5) * sw).to(dtype)
    w[0] = 0
    return x, w, torch.zeros(n, dtype=torch.int64, device="cuda")


def held(p, dtype):
    """G relative to the largest row weight, as it is held: in float16 2^15 times as large."""
    scale = 32768.0 if dtype == torch.float16 else 1.0
    return (p * scale).to(dtype).double() / scale


@pytest.mark.parametrize("n,d,v", [(2048, 2048, 131072), (40, 256, 600000)])
def test_dx_does_not_shrink_with_the_vocabulary(ops, n, d, v):
    dtype = torch.float16
    x, w, t = one_signed(1, n, d, v, dtype, 2.0 ** -5, 2.0 ** -9 * math.sqrt(2048 / d))
    one = torch.ones(1, device="cuda")
    out = ops.linear_xent(x, w, t)
    dx = ops.linear_xent_grad(x, w, t, out["lse"], one, out={"dx": torch.empty_like(x)})["dx"].double()
    xd, wd = x.double(), w.double()
    # (The target's part falls on a row of zeros.  Both roundings that the operator states are the reference's too: the values
    # lie so close together that rounding them, near a power of two, has a mean of its own.)
    p = held(torch.softmax(xd @ wd.T, 1), dtype)
    want = p @ wd
    err = float(((dx - want.to(dtype).double()) / want).mean())
    big = float((xd.abs().sum(1) * wd.amax()).max())
    # exponentials: three times a logit's error and 2^-20; sums: pieces, added up in float32 (one rounding each)
    tol = 3 * ((min(d, 1024) / 16 + 16) * 2 * U32 * big + 2.0 ** -20) + PIECE + math.ceil(v / 1024) * U32
    # values and G that fall on the other side of a rounding's border: no more than if all of them did, six deviations
    tol += 6 * 2 * HALF[dtype] / math.sqrt(3 * n * d) + 6 * HALF[dtype] / math.sqrt(3 * v)
    assert abs(err) <= tol, (err, tol)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,d,v", [(1 << 20, 64, 64), ((1 << 21) - 77, 8, 40)])
def test_dw_does_not_shrink_with_the_rows(ops, dtype, n, d, v):
    """The entries that are never a target only collect positive G; x is positive here."""
    g = gen(n)
    x = (torch.rand(n, d, generator=g, device="cuda") + 0.5).to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") * (0.1 / d)).to(dtype)
    t = torch.zeros(n, dtype=torch.int64, device="cuda")
    one = torch.full((1,), 64.0 / n, device="cuda")
    out = ops.linear_xent(x, w, t)
    dw = ops.linear_xent_grad(x, w, t, out["lse"], one, out={"dw": torch.empty_like(w)})["dw"][1:].double()
    xd, wd = x.double(), w.double()
    p = held(torch.softmax(xd @ wd.T, 1), dtype)
    want = (p.T @ xd * float(one))[1:]
    err = float(((dw - want.to(dtype).double()) / want).mean())
    big = float((xd @ wd.abs().T).max())
    tol = 3 * ((d / 16 + 16) * 2 * U32 * big + 2.0 ** -20) + PIECE + math.ceil(n / 1024) * U32
    tol += 6 * HALF[dtype] / math.sqrt(3 * d * (v - 1)) + 6 * HALF[dtype] / math.sqrt(3 * n)
    assert abs(err) <= tol, (err, tol)
