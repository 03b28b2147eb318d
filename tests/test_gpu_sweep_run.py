"""The node sweep's load: its training step against float64, its determinism, and its results through qualification."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def run():
    from paper_2605_17879_b200 import sweep_run
    return sweep_run


def test_a_step_is_the_formulas(run):
    """Lookup, loss, gradients of a table used twice, update: one step against autograd in float64 from the same bfloat16
    weights."""
    load = run.SweepStep(rows=300, width=64, vocab=500, lr=1e-2, seed=3)
    before = load.param.double()
    w = load.weights.double().requires_grad_()
    x = (w[load.tokens] * load.scale)
    x16 = x.detach().bfloat16().double()
    # the operators see x rounded to bfloat16; the gradient passes through unchanged
    xr = x + (x16 - x).detach()
    z = xr @ w.T
    loss = torch.logsumexp(z, 1) - z.gather(1, load.targets[:, None])[:, 0]
    loss.mean().backward()
    got = load.step().double()
    # a logit of 64 products: (64 / 16 + 16) steps of 2^-23 of its terms' magnitudes, twice, and the exponentials' 2^-21
    size = (xr.detach().abs() @ w.detach().abs().T).amax(1)
    assert ((got - loss.detach()).abs() <= 2 * (24 * 2.0 ** -23 * size + 2.0 ** -20) + 2.0 ** -23 * loss.detach().abs()).all()
    grad = w.grad
    # dw and dx round to bfloat16 (2^-8 of their values), G too (2^-8 of its terms), and the sum of both once more
    p = torch.exp(z.detach() - torch.logsumexp(z.detach(), 1, keepdim=True))
    G = p.clone()
    G[torch.arange(300), load.targets] -= 1
    G = G.abs() / 300
    size_dw = G.T @ xr.detach().abs()
    size_dx = G @ w.detach().abs()
    back = torch.zeros_like(grad).index_add_(0, load.tokens, size_dx * load.scale)
    assert ((load.grad.double() - grad).abs() <= 3 * 2.0 ** -8 * (size_dw + back) + 2.0 ** -8 * grad.abs() + 2.0 ** -60).all()
    # the first update moves every parameter by lr against its gradient's sign (beyond eps), after the decay
    g = load.grad.double()
    want = before * (1 - load.lr * 0.1) - load.lr * g / (g.abs() + 1e-8)
    assert ((load.param.double() - want).abs() <= 40 * 2.0 ** -24 * (load.lr + before.abs())).all()
    assert torch.equal(load.weights, load.param.bfloat16())


def test_steps_run_on_and_are_the_same_on_equal_gpus(run):
    for bits in (32, 8):
        a, b = (run.SweepStep(rows=1000, width=72, vocab=3001, state_bits=bits, seed=1).measure(6, warmup=1) for _ in range(2))
        assert a["rows"].shape == (6, 4) and bool((a["rows"] > 0).all()) and bool(a["rows"].isfinite().all())
        assert torch.equal(a["loss"], b["loss"]) and bool(a["loss"].isfinite().all())
        other = run.SweepStep(rows=1000, width=72, vocab=3001, state_bits=bits, seed=2).measure(6, warmup=1)
        assert not torch.equal(a["loss"], other["loss"])
    with pytest.raises(ValueError):
        run.SweepStep(width=60)
    with pytest.raises(ValueError):
        run.SweepStep(rows=16, width=64, vocab=100).measure(0)


def test_a_step_can_be_captured(run):
    a, b = (run.SweepStep(rows=200, width=64, vocab=300, seed=5) for _ in range(2))
    for k in (a, b):
        k.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for _ in range(3):
        graph.replay()
        b.step()
        assert torch.equal(a.loss["loss"], b.loss["loss"]) and torch.equal(a.param, b.param)
    assert a.opt.steps() == b.opt.steps() == 4


def test_measured_rows_are_qualified(run):
    """A fleet of GPUs that measured like this one, one of them a fifth slower in the tensor cores' part, fails."""
    rows = run.SweepStep(rows=512, width=128, vocab=2000).measure(16)["rows"]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    fleet = rows[None] * (1 + 0.002 * torch.randn(64, 1, 4, generator=g, device="cuda"))
    fleet[21, :, 0] *= 0.8
    out = run.qualify(fleet.float(), 8, 8, pct_ppm=50_000)       # the cut is the fourth worst: only what lies beyond it can fail
    passed = out["gpu_pass"].cpu()
    assert passed[21] == 0 and int(out["fail_mask"][21]) & 1
    assert out["node_pass"][21 // 8] == 0
    assert math.isfinite(float(out["fleet_med"][0]))
