"""Token embedding, its gradient and AdamW on the GPU against the formulas in float64.

Tolerances count roundings (u = 2^-24 for float32; half a step of the output's type for its one rounding) and are stated
beside each check."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step relative to the value
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}    # half a step near zero
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    from paper_2605_17879_b200 import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


# ---- embedding ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,width,pad", [(1, 1, 1, 0), (1, 7, 8, 0), (63, 100, 513, 0), (200, 33, 1001, 3), (1000, 5000, 64, 8), (77, 9, 4096, 0)])
def test_embed(ops, dtype, n, rows, width, pad):
    g = gen(n + width)
    store = randn(g, rows, width + pad).to(dtype)
    table = store[:, :width]
    ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
    for tokens in (ids, ids.int()):
        got = ops.embed(tokens, table, scale=1.7)["out"]
        # one float32 product and one rounding: nothing to be off by
        assert torch.equal(got, (table[ids].float() * 1.7).to(dtype))
    ops.sync_status()


def test_embed_shapes_status_and_unaligned(ops):
    g = gen(3)
    flat = randn(g, 1 + 50 * 24).bfloat16()
    table = flat[1:].view(50, 24)                      # two bytes off every alignment
    ids = torch.randint(0, 50, (4, 5), generator=g, device="cuda")
    got = ops.embed(ids, table)["out"]
    assert got.shape == (4, 5, 24) and torch.equal(got, table[ids])
    assert ops.embed(ids[:0], table)["out"].shape == (0, 5, 24)
    bad = ids.clone()
    bad[1, 2], bad[3, 4] = 50, -1
    got = ops.embed(bad, table)["out"]
    good = (bad >= 0) & (bad < 50)
    assert torch.equal(got[good], table[bad[good]]) and got[~good].isnan().all()
    with pytest.raises(ops.GuardError):
        ops.sync_status()
    ops.sync_status()                                  # cleared
    out = {"out": torch.empty(20, 24, dtype=torch.bfloat16, device="cuda"), "status": torch.zeros(1, dtype=torch.uint32, device="cuda")}
    ops.embed(bad, table, out=out)
    assert int(out["status"].item()) == ops.STATUS_INDEX
    ops.sync_status()


def ref_embed_grad(grad, ids, rows, scale, padding):
    use = ids != padding
    total = torch.zeros(rows, grad.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    total.index_add_(0, ids[use], grad[use].double())
    size.index_add_(0, ids[use], grad[use].double().abs())
    count = torch.zeros(rows, dtype=torch.float64, device="cuda").index_add_(0, ids[use], torch.ones(int(use.sum()), dtype=torch.float64, device="cuda"))
    return total * scale, size * abs(scale), count[:, None]


def check_grad(got, want, size, count, dtype):
    # count float32 additions in any grouping, a product and (accumulating) one more addition; then the rounding
    bound = (count + 2) * U32 * size * 1.01 + want.abs() * HALF[dtype] * 1.01 + TINY[dtype]
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,width,pad,kind", [
    (1, 1, 1, 0, "uniform"), (1, 70000, 8, 0, "uniform"), (64, 3, 16, 0, "uniform"), (65, 2, 1001, 0, "one"), (129, 513, 100, 4, "uniform"),
    (2048, 511, 64, 0, "zipf"), (2049, 512, 24, 0, "zipf"), (5003, 32001, 72, 1, "zipf"), (4096, 300000, 8, 0, "uniform"),
    (1500, 10, 2056, 0, "one"), (9000, 5, 40, 0, "one"), (6000, 262144, 16, 0, "ends"), (40000, 1000, 33, 0, "zipf"), (8192, 600, 8, 0, "zipf"), (8193, 600, 8, 0, "zipf"), (131073, 700, 8, 0, "zipf"),
    (300001, 1000000, 8, 0, "uniform")])
def test_embed_grad(ops, dtype, n, rows, width, pad, kind):
    g = gen(n + rows)
    grad = randn(g, n, width + pad).to(dtype)[:, :width]
    if kind == "uniform":
        ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
    elif kind == "zipf":
        ids = (rows ** torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).long().clamp(max=rows) - 1
    elif kind == "one":
        ids = torch.full((n,), rows - 1, device="cuda")
        ids[n // 2] = 0
    else:
        ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, 0, rows - 1)
    padding = int(ids[n // 3])
    for tokens, pid in ((ids, -1), (ids.int(), padding)):
        want, size, count = ref_embed_grad(grad, ids, rows, 0.5, pid)
        out = {"dtable": torch.full((rows, width), float("nan"), dtype=dtype, device="cuda")}
        got = ops.embed_grad(grad, tokens, rows, scale=0.5, padding_idx=pid, out=out)["dtable"]
        check_grad(got, want, size, count, dtype)
        assert torch.equal(got, ops.embed_grad(grad, tokens, rows, scale=0.5, padding_idx=pid)["dtable"])    # bit for bit
    base = randn(g, rows, width).to(dtype)
    kept = base.clone()
    ops.embed_grad(grad, ids, rows, scale=0.5, accumulate=True, out={"dtable": base})
    want, size, count = ref_embed_grad(grad, ids, rows, 0.5, -1)
    check_grad(base, kept.double() + want, size + kept.double().abs(), count, dtype)
    untouched = count[:, 0] == 0
    assert torch.equal(base[untouched], kept[untouched])
    ops.sync_status()


def test_embed_grad_bad_tokens_and_empty(ops):
    grad = torch.ones(6, 8, device="cuda")
    ids = torch.tensor([0, 4, -1, 3, 2 ** 40, 3], device="cuda")
    got = ops.embed_grad(grad, ids, 4)["dtable"]
    assert got.tolist() == [[1.0] * 8, [0.0] * 8, [0.0] * 8, [2.0] * 8]
    with pytest.raises(ops.GuardError):
        ops.sync_status()
    assert ops.embed_grad(grad[:0], ids[:0], 4)["dtable"].eq(0).all()
    all_pad = torch.full((6,), 2, device="cuda")
    assert ops.embed_grad(grad, all_pad, 4, padding_idx=2)["dtable"].eq(0).all()
    ops.sync_status()


def test_embed_grad_is_the_difference_quotient(ops):
    # the lookup is linear: the change of sum(out * grad) along a direction is the gradient's product with it
    g = gen(9)
    table, direction, grad = randn(g, 40, 24), randn(g, 40, 24), randn(g, 300, 24)
    ids = torch.randint(0, 40, (300,), generator=g, device="cuda")
    def value(t):
        return (ops.embed(ids, t, scale=0.7)["out"].double() * grad.double()).sum()
    d = ops.embed_grad(grad, ids, 40, scale=0.7)["dtable"].double()
    quotient = (value(table + direction) - value(table - direction)) / 2
    # each of 2 x 7200 products off by the roundings of table +- direction and of the scaling: 2 u of values of size below 10
    assert abs(float(quotient - (d * direction.double()).sum())) <= 2 * 7200 * 2 * U32 * 10 * 4


def test_embed_streams_and_graph(ops):
    g = gen(12)
    table, grad = randn(g, 500, 64).bfloat16(), randn(g, 3000, 64).bfloat16()
    ids = torch.randint(0, 500, (3000,), generator=g, device="cuda")
    out = ops.embed(ids, table)
    back = ops.embed_grad(grad, ids, 500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other, other_back = ops.embed(ids, table), ops.embed_grad(grad, ids, 500)
    side.synchronize()
    assert torch.equal(other["out"], out["out"]) and torch.equal(other_back["dtable"], back["dtable"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.embed(ids, table, out=out)
        ops.embed_grad(grad, ids, 500, out=back)
    for seed in (1, 2):
        h = gen(seed)
        table.copy_(randn(h, 500, 64))
        grad.copy_(randn(h, 3000, 64))
        ids.copy_(torch.randint(0, 500, (3000,), generator=h, device="cuda"))
        graph.replay()
        got, got_back = out["out"].clone(), back["dtable"].clone()
        assert torch.equal(got, ops.embed(ids, table)["out"]) and torch.equal(got_back, ops.embed_grad(grad, ids, 500)["dtable"])


# ---- AdamW -------------------------------------------------------------------------------------------------------------

def flat_of(tensors, block):
    total = sum((t.numel() + block - 1) // block * block for t in tensors)
    flat, inside, at = torch.zeros(total, dtype=torch.float64, device="cuda"), torch.zeros(total, dtype=torch.bool, device="cuda"), 0
    for t in tensors:
        flat[at:at + t.numel()] = t.double().reshape(-1)
        inside[at:at + t.numel()] = True
        at += (t.numel() + block - 1) // block * block
    return flat, inside


def scale_of(top):
    """The power of two by which top comes to lie in (224, 448]."""
    return 2.0 ** torch.ceil(torch.log2(top.double() / 448)).float()


def step_of_e4m3(y):
    """Distance of the 8-bit values around y >= 0."""
    return torch.where(y < 2.0 ** -6, 2.0 ** -9, 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3))


SHAPES = [[(1,)], [(256,)], [(255,), (0,), (257,)], [(300, 7), (1,), (1023,), (8,), (64, 64), (2049,)], [(7,)] * 70, [(513, 1001), (3,), (100000,)]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype,ctype", [(torch.bfloat16, torch.bfloat16), (torch.float16, None), (torch.float32, torch.float16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: "%dx%s" % (len(s), s[0]))
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_step(ops, bits, gtype, ctype, shapes, shift):
    g = gen(len(shapes) + shift)
    def tensor(shape, scale, dtype):
        n = math.prod(shape)
        return (randn(g, n + shift) * scale).to(dtype)[shift:].view(shape)     # shift 1: off every vector's alignment
    params = [tensor(s, 0.02, torch.float32) for s in shapes]
    grads = [tensor(s, 1e-3, gtype) for s in shapes]
    copies = [tensor(s, 1.0, ctype) for s in shapes] if ctype is not None else None
    decay = [0.1 * (i % 2) for i in range(len(shapes))]
    b1, b2, eps, lr, gs, at = 0.9, 0.95, 1e-8, 3e-3, 0.5, 7
    opt = ops.AdamW(params, grads, betas=(b1, b2), eps=eps, weight_decay=decay, state_bits=bits, copies=copies, step=at, seed=5)
    p0, inside = flat_of(params, ops.BLOCK)
    gr, _ = flat_of(grads, ops.BLOCK)
    wd, _ = flat_of([torch.full(s, d) for s, d in zip(shapes, decay)], ops.BLOCK)
    mark = {}
    for name, scale in (("m", 3e-4), ("v", 1e-3)):
        x = randn(g, len(p0)) * scale
        if name == "v":
            x = x.abs() + 1e-4
        if bits == 32:
            opt.state[name].copy_(x if name == "m" else x * x)
        else:
            x = x if name == "m" else x * x
            s = scale_of(x.view(-1, ops.BLOCK).abs().amax(1))
            opt.state[name].copy_((x.view(-1, ops.BLOCK) / s[:, None]).view(-1))
            opt.state[name + "_scale"].copy_(s)
        mark[name] = opt.state[name].clone()
    def held(name):
        x = opt.state[name].double()
        return x if bits == 32 else x * opt.state[name + "_scale"].double().repeat_interleave(ops.BLOCK)
    m0, v0 = held("m"), held("v")
    opt.step(lr, grad_scale=torch.tensor([gs], device="cuda"))
    t = at + 1
    assert opt.steps() == t
    g1 = gr * gs
    m, v = b1 * m0 + (1 - b1) * g1, b2 * v0 + (1 - b2) * g1 * g1
    den = v.sqrt() / math.sqrt(1 - b2 ** t) + eps
    rate = lr / (1 - b1 ** t)
    p = p0 * (1 - lr * wd) - rate * m / den
    p1, _ = flat_of(params, ops.BLOCK)
    # m: the constants, products and the sum round once each: 6 u of its terms
    mtol = 6 * U32 * (b1 * m0.abs() + (1 - b1) * g1.abs()) + 2.0 ** -148
    # v: likewise, with a square: 8 u of its terms, all positive
    vrel = 8 * U32
    # the update: m's error, and relatively: den 4 u from v, then root, quotient, constant, sum, eps; the rate, quotient, product
    ptol = rate / den * mtol + (rate * m / den).abs() * 14 * U32 + 3 * U32 * p0.abs() + U32 * p.abs() + 2.0 ** -148
    assert ((p1 - p).abs() <= ptol)[inside].all()
    assert torch.equal(p1[~inside], p0[~inside])
    if copies is not None:
        for c, q in zip(copies, params):
            assert torch.equal(c, q.to(ctype))
    if bits == 32:
        assert ((held("m") - m).abs() <= mtol)[inside].all()
        assert ((held("v") - v).abs() <= vrel * v + 2.0 ** -148)[inside].all()
    else:
        for name, x, tol in (("m", m, mtol), ("v", v, vrel * v)):
            x = torch.where(inside, x, 0.0)
            top = x.view(-1, ops.BLOCK).abs().amax(1)
            scale = opt.state[name + "_scale"].double()
            wide = 1 + 16 * U32
            assert ((top <= 448 * scale * wide) & (top * wide > 224 * scale))[top > 0].all() and (torch.frexp(scale).mantissa == 0.5).all()
            each = scale.repeat_interleave(ops.BLOCK)
            # rounded to a neighbour among the 8-bit values of this scale
            assert ((held(name) - x).abs() <= step_of_e4m3(x.abs() / each * wide) * each + tol)[inside].all()
    for name in ("m", "v"):                                 # what lies behind a tensor's end
        assert torch.equal(opt.state[name].view(torch.uint8 if bits == 8 else torch.int32)[~inside], mark[name].view(torch.uint8 if bits == 8 else torch.int32)[~inside])
    opt.close()


def test_adamw_8bit_rounding_is_unbiased(ops):
    """What is held has the mean of what was computed: the dithering's error over 2^20 values is a mean of independent terms
    of at most a step each (variance at most 1/4 step^2): six standard deviations are 3 steps / sqrt(n)."""
    n = 1 << 20
    g = gen(4)
    p, grad = torch.zeros(n, device="cuda"), randn(g, n) * 1e-3
    opt = ops.AdamW([p], [grad], betas=(0.0, 0.0), state_bits=8, seed=77)     # m = g, v = g^2
    opt.step(0.0)
    scale = {k: opt.state[k + "_scale"].double().repeat_interleave(ops.BLOCK) for k in ("m", "v")}
    for name, x in (("m", grad.double()), ("v", (grad * grad).double())):
        y = x.abs() / scale[name]
        err = (opt.state[name].double().abs() - y) / step_of_e4m3(y)
        # (second moments below one smallest step are held as one step: left out)
        ok = y >= (2.0 ** -9 if name == "v" else 0.0)
        for part in (ok, ok & (y < 2.0 ** -6), ok & (y > 100), ok & (torch.arange(n, device="cuda") % 2 == 0)):
            k = int(part.sum())
            if k:                                   # (16 random bits: 2^-17 of a step of bias)
                assert abs(float(err[part].mean())) <= 3 / math.sqrt(k) + 2.0 ** -16
    # another step number, other bits; the same, the same
    one = opt.state["m"].clone().view(torch.uint8)
    opt.step(0.0)
    assert not torch.equal(one, opt.state["m"].view(torch.uint8))
    again = ops.AdamW([p], [grad], betas=(0.0, 0.0), state_bits=8, seed=77)
    again.step(0.0)
    assert torch.equal(one, again.state["m"].view(torch.uint8))
    other = ops.AdamW([p], [grad], betas=(0.0, 0.0), state_bits=8, seed=78)
    other.step(0.0)
    assert not torch.equal(one, other.state["m"].view(torch.uint8))


def test_adamw_8bit_tracks_a_slow_mean(ops):
    """An exponential mean whose steps are far below a step of 8 bits still moves: rounding to nearest would hold it."""
    n = 4096
    p, grad = torch.zeros(n, device="cuda"), torch.full((n,), 1.0, device="cuda")
    opt = ops.AdamW([p], [grad], betas=(0.99, 0.999), state_bits=8, seed=3)
    grad[::256] = 4.0                                       # each block's largest: the others lie inside the 8-bit range
    for _ in range(400):
        opt.step(0.0)
    v = opt.state["v"].float() * opt.state["v_scale"].repeat_interleave(256)
    want = 1 - 0.999 ** 400
    inner = torch.arange(n, device="cuda") % 256 != 0
    # an update moves v by at most 0.001, up a step with that over the step as its probability: 400 steps of at most 1/8 of
    # v <= 0.33 have a variance of at most 400 * 0.001 * 0.041; six deviations of the mean of 4 080 such values, over want
    assert abs(float(v[inner].mean()) / want - 1) < 6 * math.sqrt(400 * 0.001 * 0.041 / 4080) / want
    assert float(v[inner].std()) / want < 0.45


def test_adamw_zero_gradient_of_a_small_state_stays_bounded(ops):
    """A state far below its block's largest keeps a second moment of one smallest step, so a parameter whose gradient stops does not
    jump by m / eps."""
    p, grad = torch.zeros(256, device="cuda"), torch.full((256,), 1e-9, device="cuda")
    grad[0] = 1.0
    opt = ops.AdamW([p], [grad], state_bits=8)
    for k in range(50):
        if k == 10:
            grad.zero_()
        opt.step(1e-3)
    assert (opt.state["v"].float() > 0).all()
    assert p.isfinite().all() and float(p.abs().max()) < 50 * 1e-3 * 40


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_graph_counts_steps_and_reads_lr(ops, bits):
    g = gen(8)
    start, grads = [randn(g, 1000), randn(g, 33)], [randn(g, 1000), randn(g, 33)]
    lr = torch.tensor([1e-2], device="cuda")
    runs = []
    for captured in (False, True):
        params = [p.clone() for p in start]
        opt = ops.AdamW(params, grads, weight_decay=0.1, state_bits=bits, seed=1)
        lr.fill_(1e-2)
        opt.step(lr)
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                opt.step(lr)
        for k in range(3):
            lr.fill_(1e-2 / (k + 2))
            graph.replay() if captured else opt.step(lr)
        assert opt.steps() == 4
        runs.append((params, {k: v.clone() for k, v in opt.state.items()}))
        opt.close()
    for a, b in zip(runs[0][0], runs[1][0]):
        assert torch.equal(a, b)
    for k in runs[0][1]:
        assert torch.equal(runs[0][1][k].view(torch.uint8), runs[1][1][k].view(torch.uint8))


def test_adamw_non_finite_gradients_stay_where_they_are(ops):
    p, grad = torch.ones(512, device="cuda"), torch.ones(512, device="cuda")
    grad[3], grad[300] = float("nan"), float("nan")
    opt = ops.AdamW([p], [grad], state_bits=32)
    opt.step(1e-2)
    bad = torch.zeros(512, dtype=torch.bool, device="cuda")
    bad[3] = bad[300] = True
    assert p[bad].isnan().all() and p[~bad].isfinite().all()
    p8 = torch.ones(512, device="cuda")
    opt = ops.AdamW([p8], [grad], state_bits=8)
    opt.step(1e-2)
    assert p8[bad].isnan().all() and p8[~bad].isfinite().all()
    m = opt.state["m"].float() * opt.state["m_scale"].repeat_interleave(256)
    assert m[bad].isnan().all() and ((m[~bad] - 0.1).abs() < 0.1 / 8).all()       # a neighbour of 0.1 in 8 bits
