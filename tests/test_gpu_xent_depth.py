"""What long depths may cost the cross entropy's gradients: nothing that grows with the depth.

The tensor cores cut off what an accumulator's last bit cannot hold, so an accumulation of one-signed terms shrinks with every
step of 16.  u = 2^-24; h half a step of the inputs' type relative to the value (bfloat16 2^-8, float16 2^-11)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


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
