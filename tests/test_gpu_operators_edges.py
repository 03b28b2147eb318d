"""Calls at the operators' edges on the GPU: values, streams, captures and threads that the ordinary tests do not meet."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2605_17879_b200 import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("weight", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_weight_that_is_not_finite_reaches_its_row_of_dx_alone(ops, dtype, weight):
    n, d, v = 200, 64, 500
    g = gen(1)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") * 0.25).to(dtype)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    grad = torch.full((n,), 1e-4, device="cuda")        # (times a probability of 1/500: below float16's smallest step)
    out = ops.linear_xent(x, w, t)
    others = torch.arange(n, device="cuda") != 17
    want = ops.linear_xent_grad(x, w, torch.where(others, t, -100), out["lse"], grad)["dx"]
    grad[17] = weight
    got = ops.linear_xent_grad(x, w, t, out["lse"], grad)["dx"]
    assert torch.equal(got[others], want[others])        # the same arithmetic in another row of the tile
    assert not got[17].isfinite().any()
    # all of them: nothing to be relative to
    assert not ops.linear_xent_grad(x, w, t, out["lse"], torch.full((1,), weight, device="cuda"))["dx"].isfinite().any()
