"""Softmax cross entropy of a vocabulary product and its gradients against float64.

Tolerances count roundings: u = 2^-24; h half a step of the inputs' type relative to the value (bfloat16 2^-8, float16 2^-11)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def ops():
    from paper_2605_17879_b200 import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def inputs(seed, n, d, v, dtype, ignored=0.0, pad=0, std=2.0):
    g = gen(seed)
    x = torch.randn(n, d + pad, generator=g, device="cuda").to(dtype)[:, :d]
    w = (torch.randn(v, d + pad, generator=g, device="cuda") * (std / math.sqrt(d))).to(dtype)[:, :d]
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    gone = torch.rand(n, generator=g, device="cuda") < ignored
    t[gone] = -100
    grad = torch.rand(n, generator=g, device="cuda") / n
    return x, w, t, grad


def reference(x, w, t, grad):
    """Loss, log sums and gradients in float64, and the sizes that their errors go by."""
    x, w = x.double(), w.double()
    keep = t != -100
    at = torch.where(keep, t, 0)[:, None]
    z = x @ w.T
    size = x.abs() @ w.abs().T                                   # what a logit's rounding goes by
    lse = torch.logsumexp(z, 1)
    loss = (lse - z.gather(1, at)[:, 0]) * keep
    p = torch.exp(z - lse[:, None])
    big = size.amax(1) if len(w) else size.sum(1)
    G = p.clone()
    G.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float64))
    # |error of G| relative to p: a logit's and the log sum's error, and the exponential
    gk = (grad.double() * keep)[:, None]
    return dict(loss=loss, lse=lse * keep, dx=(G * gk) @ w, dw=(G * gk).T @ x, big=big * keep, P=p * gk, G=G * gk, x=x, w=w, keep=keep)


def check_forward(out, ref, d):
    # A logit: d products summed in float32 in steps of 16 (the tensor cores keep at least 23 bits of each partial sum, cut
    # off rather than rounded): (d / 16 + 16) steps of 2 u of the sum of magnitudes.  The log sum: the largest such error,
    # the exponents' rounding (products with log2 e: 4 u of the logit's size), exponentials and sums (2^-21), the logarithm.
    tol = (d / 16 + 16) * 2 * U32 * ref["big"] + 8 * U32 * ref["big"] + 2.0 ** -21 + 4 * U32 * ref["lse"].abs()
    tol = tol * ref["keep"]
    assert ((out["lse"].double() - ref["lse"]).abs() <= tol).all()
    assert ((out["loss"].double() - ref["loss"]).abs() <= 2 * tol + U32 * ref["loss"].abs()).all()


def check_grads(out, ref, grad, d, n, v, dtype):
    h = HALF[dtype]
    rel = 3 * ((d / 16 + 16) * 2 * U32 * ref["big"] + 2.0 ** -20)[:, None]     # of exp(z - lse): logit, log sum and exponential
    # G: that of its exponential, two float32 roundings of its row's weight, and one to the inputs' type; in float16 also
    # half a smallest step, 2^-25, relative to 2^15 times the largest weight
    top = grad.abs().max().double() if dtype == torch.float16 else 0.0
    gerr = ref["P"] * rel + ref["G"].abs() * (h + 4 * U32) + top * 2.0 ** -40
    for name, err, size, want, depth in (("dx", gerr @ ref["w"].abs(), ref["G"].abs() @ ref["w"].abs(), ref["dx"], v),
                                         ("dw", gerr.T @ ref["x"].abs(), ref["G"].abs().T @ ref["x"].abs(), ref["dw"], n)):
        tol = (err + (depth / 16 + 16) * 2 * U32 * size) * 1.01 + want.abs() * h * 1.01 + TINY[dtype]
        bad = (out[name].double() - want).abs() > tol
        assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[0].tolist())


CASES = [  # rows, width, vocab, ignored, row padding
    (1, 8, 1, 0.0, 0), (1, 64, 100, 0.0, 0), (3, 72, 257, 0.0, 8), (48, 512, 1000, 0.0, 0), (128, 128, 256, 0.3, 0), (129, 136, 513, 0.0, 0),
    (200, 64, 31, 0.5, 0), (257, 1000, 2049, 0.3, 16), (300, 8, 5000, 0.1, 0), (1003, 264, 3001, 0.3, 0), (640, 2048, 777, 0.0, 0), (64, 256, 40000, 0.0, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,d,v,ignored,pad", CASES)
def test_loss_and_gradients(ops, dtype, n, d, v, ignored, pad):
    x, w, t, grad = inputs(n + v, n, d, v, dtype, ignored, pad)
    ref = reference(x, w, t, grad)
    for targets in (t, t.int()):
        out = ops.linear_xent(x, w, targets)
        ops.sync_status()
        check_forward(out, ref, d)
        back = ops.linear_xent_grad(x, w, targets, out["lse"], grad)
        ops.sync_status()
        check_grads(back, ref, grad, d, n, v, dtype)
    again = ops.linear_xent_grad(x, w, t, out["lse"], grad)
    assert torch.equal(again["dx"], back["dx"]) and torch.equal(again["dw"], back["dw"])     # bit for bit
    assert torch.equal(ops.linear_xent(x, w, t)["loss"], out["loss"])
    only = {"dw": torch.empty_like(w.contiguous())}
    assert torch.equal(ops.linear_xent_grad(x, w, t, out["lse"], grad, out=only)["dw"], back["dw"])
    only = {"dx": torch.empty_like(x.contiguous()), "dw": None}
    assert torch.equal(ops.linear_xent_grad(x, w, t, out["lse"], grad, out=only)["dx"], back["dx"])
