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


@pytest.mark.parametrize("d", [1024, 1032, 2056, 4096])
def test_depth_beyond_one_pass(ops, d):
    x, w, t, grad = inputs(d, 150, d, 300, torch.bfloat16)
    ref = reference(x, w, t, grad)
    out = ops.linear_xent(x, w, t)
    check_forward(out, ref, d)
    # the passes keep the log sum within 1e-6 of itself, over all rows
    assert float((out["lse"].double() - ref["lse"]).norm() / ref["lse"].norm()) < 1e-6
    check_grads(ops.linear_xent_grad(x, w, t, out["lse"], grad), ref, grad, d, 150, 300, torch.bfloat16)


def test_vocabulary_in_several_pieces(ops):
    # so many rows that a piece of G is 256 entries wide: three pieces, the last one partial
    n, d, v = (1 << 20) - 77, 8, 600
    x, w, t, grad = inputs(5, n, d, v, torch.bfloat16, ignored=0.25)
    ref = reference(x, w, t, grad)
    out = ops.linear_xent(x, w, t)
    check_forward(out, ref, d)
    check_grads(ops.linear_xent_grad(x, w, t, out["lse"], grad), ref, grad, d, n, v, torch.bfloat16)
    ops.sync_status()


def test_piece_boundaries_of_a_large_vocabulary(ops):
    # 2 048 rows and 150 000 entries: two pieces; a few columns of dw on either side of the border, and all of dx
    n, d, v = 2048, 64, 150000
    x, w, t, grad = inputs(6, n, d, v, torch.float16)
    ref = reference(x, w, t, grad)
    out = ops.linear_xent(x, w, t)
    check_forward(out, ref, d)
    check_grads(ops.linear_xent_grad(x, w, t, out["lse"], grad), ref, grad, d, n, v, torch.float16)


@pytest.mark.parametrize("n", [100, 400])
def test_ignored_rows_reach_nothing(ops, n):
    x, w, t, grad = inputs(n, n, 64, 300, torch.bfloat16, ignored=0.5)
    clean = ops.linear_xent(x, w, t)
    back = ops.linear_xent_grad(x, w, t, clean["lse"], grad)
    gone = t == -100
    assert gone.any() and (clean["loss"][gone] == 0).all() and (clean["lse"][gone] == 0).all() and (back["dx"][gone] == 0).all()
    dirty = x.clone()
    dirty[gone] = float("nan")
    dirty[gone.nonzero()[0]] = float("inf")
    g2 = torch.where(gone, float("nan"), grad)
    out = ops.linear_xent(dirty, w, t)
    assert torch.equal(out["loss"], clean["loss"]) and torch.equal(out["lse"], clean["lse"])
    b2 = ops.linear_xent_grad(dirty, w, t, out["lse"], g2)
    assert torch.equal(b2["dx"], back["dx"]) and torch.equal(b2["dw"], back["dw"])
    # another number for "ignored"
    t7 = torch.where(gone, 7, t)
    t7[~gone & (t == 7)] = 8
    out = ops.linear_xent(x, w, t7, ignore_index=7)
    assert ((out["loss"] == 0) == (t7 == 7)).all()


@pytest.mark.parametrize("n", [5, 300])
def test_all_rows_ignored_and_no_rows(ops, n):
    x, w, t, grad = inputs(1, n, 64, 300, torch.bfloat16)
    t[:] = -100
    out = ops.linear_xent(x, w, t)
    assert (out["loss"] == 0).all() and (out["lse"] == 0).all()
    nan = {"dx": torch.full_like(x, float("nan")), "dw": torch.full_like(w, float("nan"))}
    back = ops.linear_xent_grad(x, w, t, out["lse"], grad, out=nan)
    assert (back["dx"] == 0).all() and (back["dw"] == 0).all()
    out = ops.linear_xent(x[:0], w, t[:0])
    assert out["loss"].shape == (0,)
    back = ops.linear_xent_grad(x[:0], w, t[:0], out["lse"], grad[:0], out={"dw": torch.full_like(w, float("nan"))})
    assert (back["dw"] == 0).all()
    ops.sync_status()


@pytest.mark.parametrize("n", [60, 260])
def test_targets_outside_the_vocabulary(ops, n):
    x, w, t, grad = inputs(2, n, 64, 300, torch.bfloat16)
    bad = t.clone()
    bad[3], bad[n - 1], bad[10] = 300, -1, 2 ** 40
    wrong = bad != t
    status = torch.zeros(1, dtype=torch.uint32, device="cuda")
    out = {"loss": torch.empty(n, device="cuda"), "lse": torch.empty(n, device="cuda"), "status": status}
    ops.linear_xent(x, w, bad, out=out)
    assert int(status.item()) == ops.STATUS_INDEX
    good = ops.linear_xent(x, w, torch.where(wrong, -100, t))
    assert out["loss"][wrong].isnan().all() and (out["lse"][wrong] == 0).all() and torch.equal(out["loss"][~wrong], good["loss"][~wrong])
    ops.sync_status()
    back = ops.linear_xent_grad(x, w, bad, out["lse"], grad)
    with pytest.raises(ops.GuardError):
        ops.sync_status()
    want = ops.linear_xent_grad(x, w, torch.where(wrong, -100, t), good["lse"], grad)
    assert torch.equal(back["dx"], want["dx"]) and torch.equal(back["dw"], want["dw"])


def test_one_weight_for_all_rows_and_odd_weights(ops):
    x, w, t, _ = inputs(3, 200, 128, 500, torch.bfloat16)
    out = ops.linear_xent(x, w, t)
    one = torch.tensor([0.005], device="cuda")
    a = ops.linear_xent_grad(x, w, t, out["lse"], one)
    b = ops.linear_xent_grad(x, w, t, out["lse"], one.expand(200).contiguous())
    assert torch.equal(a["dx"], b["dx"]) and torch.equal(a["dw"], b["dw"])
    # weights of either sign, zeros, and sizes far apart; all zero; tiny
    for grad in (torch.randn(200, generator=gen(1), device="cuda") * 10.0 ** torch.randint(-6, 3, (200,), generator=gen(2), device="cuda"),
                 torch.zeros(200, device="cuda"), torch.full((200,), -1e-20, device="cuda")):
        grad[::7] = 0
        for dtype in (torch.bfloat16, torch.float16):
            xd, wd = x.to(dtype), w.to(dtype)
            ref = reference(xd, wd, t, grad)
            o = ops.linear_xent(xd, wd, t)
            back = ops.linear_xent_grad(xd, wd, t, o["lse"], grad)
            ref["P"], big = ref["P"].abs(), ref["big"]
            check_grads(back, ref, grad, 128, 200, 500, dtype)


def test_confident_and_far_logits(ops):
    # a target far above all others (probability 1 to the last bit), and logits of hundreds of either sign
    n, d, v = 150, 64, 400
    x, w, t, grad = inputs(4, n, d, v, torch.bfloat16, std=60.0)
    ref = reference(x, w, t, grad)
    out = ops.linear_xent(x, w, t)
    assert out["loss"].isfinite().all()
    check_forward(out, ref, d)
    top = (x.double() @ w.double().T).argmax(1)
    out = ops.linear_xent(x, w, top)
    ref = reference(x, w, top, grad)
    check_forward(out, ref, d)
    check_grads(ops.linear_xent_grad(x, w, top, out["lse"], grad), ref, grad, d, n, v, torch.bfloat16)


def test_infinite_logits_are_not_hidden(ops):
    x, w, t, grad = inputs(8, 140, 64, 300, torch.bfloat16)
    w[5] = float("inf")                          # the logit of entry 5 is infinite or NaN in every row
    out = ops.linear_xent(x, w, t)
    assert not out["loss"].isfinite().any()
    x2, w2, t2, _ = inputs(8, 140, 64, 300, torch.bfloat16)
    x2[3] = float("nan")
    out = ops.linear_xent(x2, w2, t2)
    assert out["loss"][3].isnan() and out["loss"].isnan().sum() == 1


def test_gradient_is_the_difference_quotient(ops):
    # the loss along a direction of float16 steps, in float64 from the operator's own losses
    x, w, t, grad = inputs(11, 96, 32, 200, torch.float16)
    x, w = (x * 16).round() / 16, (w * 64).round() / 64                  # steps below are exact
    dirx = torch.randint(-1, 2, x.shape, generator=gen(1), device="cuda").half() / 16
    dirw = torch.randint(-1, 2, w.shape, generator=gen(2), device="cuda").half() / 64
    def value(k):
        return float((ops.linear_xent(x + k * dirx, w + k * dirw, t)["loss"].double() * grad.double()).sum())
    out = ops.linear_xent(x, w, t)
    back = ops.linear_xent_grad(x, w, t, out["lse"], grad)
    slope = float((back["dx"].double() * dirx.double()).sum() + (back["dw"].double() * dirw.double()).sum())
    # the fourth-order quotient of the same steps in float64 says what steps of this size leave, the rest is rounding
    def exact(k):
        return float((reference((x + k * dirx).double(), (w + k * dirw).double(), t, grad)["loss"] * grad.double()).sum())
    left = abs((exact(1) - exact(-1)) / 2 - float((reference(x, w, t, grad)["dx"] * dirx.double()).sum() + (reference(x, w, t, grad)["dw"] * dirw.double()).sum()))
    quotient = (value(1) - value(-1)) / 2
    size = float((back["dx"].double() * dirx.double()).abs().sum() + (back["dw"].double() * dirw.double()).abs().sum())
    assert abs(quotient - slope) <= left + size * 2 * HALF[torch.float16] + 96 * 2.0 ** -18 * float(grad.max())


def test_streams_graph_and_workspaces(ops):
    n, d, v = 300, 64, 700
    x, w, t, grad = inputs(12, n, d, v, torch.bfloat16, ignored=0.2)
    out = ops.linear_xent(x, w, t)
    back = ops.linear_xent_grad(x, w, t, out["lse"], grad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):           # two calls at once, each with a workspace of its own
        other = ops.linear_xent(x, w, t)
        other_back = ops.linear_xent_grad(x, w, t, other["lse"], grad)
    again = ops.linear_xent_grad(x, w, t, out["lse"], grad)
    side.synchronize()
    assert torch.equal(other["loss"], out["loss"])
    for k in ("dx", "dw"):
        assert torch.equal(other_back[k], back[k]) and torch.equal(again[k], back[k])
    ws = [torch.empty(int(ops.lib().guard_linear_xent_workspace_bytes(n, d, v, g)), dtype=torch.uint8, device="cuda").fill_(255) for g in (0, 1)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.linear_xent(x, w, t, workspace=ws[0], out=out)
        ops.linear_xent_grad(x, w, t, out["lse"], grad, workspace=ws[1], out=back)
    for seed, ignored in ((1, 0.0), (2, 0.6), (3, 1.0)):
        for a, b in zip((x, w, t, grad), inputs(seed, n, d, v, torch.bfloat16, ignored)):
            a.copy_(b)
        for k in ws:
            k.fill_(255)                     # what an earlier call left says nothing
        graph.replay()
        fresh = ops.linear_xent(x, w, t)
        fresh_back = ops.linear_xent_grad(x, w, t, fresh["lse"], grad)
        assert torch.equal(out["loss"], fresh["loss"]) and torch.equal(out["lse"], fresh["lse"])
        assert torch.equal(back["dx"], fresh_back["dx"]) and torch.equal(back["dw"], fresh_back["dw"])


def test_binding_refusals_on_the_gpu(ops):
    x, w, t, grad = inputs(13, 20, 64, 100, torch.bfloat16)
    lse = torch.zeros(20, device="cuda")
    for bad in (dict(x=x.half()), dict(x=x.float(), w=w.float()), dict(w=w[:, :32]), dict(t=t[:10]), dict(t=t.float()), dict(x=x[:, ::2], w=w[:, ::2]), dict(x=x[0]),
                dict(w=w.cpu()), dict(x=x.t().contiguous().t(), w=w), dict(x=x[:1].expand(20, 64))):
        a = dict(x=x, w=w, t=t)
        a.update(bad)
        with pytest.raises(ValueError):
            ops.linear_xent(a["x"], a["w"], a["t"])
        with pytest.raises(ValueError):
            ops.linear_xent_grad(a["x"], a["w"], a["t"], lse, grad)
    for bad in (dict(x=x[:, :60].contiguous(), w=w[:, :60].contiguous()), dict(x=torch.empty(20, 65, dtype=torch.bfloat16, device="cuda")[:, 1:], w=w)):
        with pytest.raises(ops.GuardError):
            ops.linear_xent(bad["x"], bad["w"], t)
    with pytest.raises(ValueError):
        ops.linear_xent_grad(x, w, t, lse[:10], grad)
    with pytest.raises(ValueError):
        ops.linear_xent_grad(x, w, t, lse, grad.double())
    with pytest.raises(ops.GuardError):
        ops.linear_xent_grad(x, w, t, lse, grad, out={})
    with pytest.raises(ops.GuardError):
        ops.linear_xent(x, w, t, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ops.linear_xent(x, w, t, out={"loss": lse})
    with pytest.raises(ValueError):
        ops.embed(t.float(), w)
    with pytest.raises(ValueError):
        ops.embed(t, w[:, ::2])
    with pytest.raises(ValueError):
        ops.embed_grad(x, t[:5], 100)
    with pytest.raises(ValueError):
        ops.embed_grad(x, t, 100, accumulate=True)
    with pytest.raises(ops.GuardError):
        ops.embed_grad(x, t, -1)
    with pytest.raises(ops.GuardError):
        ops.embed_grad(x, t, 100, padding_idx=100)
    with pytest.raises(ops.GuardError):
        ops.embed(t, w, out={"out": w[:20]})
