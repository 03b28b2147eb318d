"""Measured calls of the training-step operators, each beside its plain form.

Three families, which one training step uses in a row: the token embedding and its gradient, the softmax cross
entropy of a vocabulary product with its gradients, and the AdamW update of all parameters.  A case is one call
(or the two calls of a loss and its gradients).  `own` says whether run() makes the framework's calls or the
elementary torch operations that define them.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}

# AdamW's constants, as training runs use them
BETA1, BETA2, EPS, DECAY, LR, AT_STEP, SEED = 0.9, 0.95, 1e-8, 0.1, 3e-4, 1000, 12345
BLOCK = 256             # parameters to a scale of the 8-bit states; every tensor starts on such a block


def listed():
    return [
        # Scoring one short sequence: a few rows, a small vocabulary; launches are what counts.
        dict(op="xent", name="xent_eval_short", rows=48, width=512, vocab=8192, type="bf16", ignored=0.0, grads=False),
        # Evaluation of a batch under a large vocabulary: the loss alone.
        dict(op="xent", name="xent_eval_batch", rows=4096, width=1024, vocab=65536, type="bf16", ignored=0.0, grads=False),
        # Fine-tuning: prompts are masked, no size is a multiple of a tile.
        dict(op="xent", name="xent_train_ragged", rows=1003, width=1000, vocab=32001, type="fp16", ignored=0.3, grads=True),
        # One training step's micro-batch.
        dict(op="xent", name="xent_train", rows=4096, width=2048, vocab=50000, type="bf16", ignored=0.02, grads=True),
        # The same of a wide model with a large vocabulary, where the logits alone would take gigabytes.
        dict(op="xent", name="xent_train_large", rows=8192, width=4096, vocab=131072, type="bf16", ignored=0.0, grads=True),
        # The lookup of a short prompt: latency.
        dict(op="embed", name="embed_short", tokens=64, width=512, vocab=8192, type="bf16", pads=0.0, grads=False),
        # The lookup of a training batch.
        dict(op="embed", name="embed_batch", tokens=16384, width=2048, vocab=65536, type="bf16", pads=0.0, grads=False),
        # The gradient of a padded batch in 32 bits, odd sizes.
        dict(op="embed", name="embed_grad_ragged", tokens=5003, width=1001, vocab=32001, type="fp32", pads=0.2, grads=True),
        # The gradient of a large batch: frequent tokens occur thousands of times.
        dict(op="embed", name="embed_grad_batch", tokens=65536, width=2048, vocab=131072, type="bf16", pads=0.0, grads=True),
        # The parameters of a small network: many small tensors, one launch.
        dict(op="adamw", name="adamw_small", layers=2, width=101, vocab=301, bits=32, type="fp32", copy=False),
        # Parameters of a middle-sized model, states in 32 bits, the weights' 16-bit copy written in the same pass.
        dict(op="adamw", name="adamw_32", layers=12, width=1024, vocab=65536, bits=32, type="bf16", copy=True),
        # A larger one with 8-bit states.
        dict(op="adamw", name="adamw_8", layers=8, width=2048, vocab=50000, bits=8, type="bf16", copy=True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["xent", "xent", "embed", "adamw"])
    if op == "xent":
        case = dict(op=op, rows=_log_uniform(rng, 1, 8192), width=8 * _log_uniform(rng, 8, 512),
                    vocab=_log_uniform(rng, 100, 131072), type=rng.choice(["bf16", "bf16", "fp16"]),
                    ignored=rng.choice([0.0, 0.0, 0.1, 0.5]), grads=rng.random() < 0.65)
        return case
    if op == "embed":
        return dict(op=op, tokens=_log_uniform(rng, 1, 65536), width=_log_uniform(rng, 16, 2048),
                    vocab=_log_uniform(rng, 100, 131072), type=rng.choice(["bf16", "fp16", "fp32"]),
                    pads=rng.choice([0.0, 0.0, 0.2]), grads=rng.random() < 0.65)
    case = dict(op=op, layers=_log_uniform(rng, 1, 16), width=_log_uniform(rng, 32, 2048), vocab=_log_uniform(rng, 100, 65536),
                bits=rng.choice([32, 8]), type=rng.choice(["bf16", "fp16", "fp32"]), copy=rng.random() < 0.6)
    while sum(_sizes(case)) > 400_000_000:
        case["layers"] = max(1, case["layers"] // 2)
        case["width"] = case["width"] * 3 // 4
    if case["type"] == "fp32":
        case["copy"] = False
    return case


def _sizes(case):
    """Elements of each parameter tensor: an embedding, a vector, and per layer two vectors and three matrices."""
    d = case["width"]
    return [case["vocab"] * d, d] + [d, d * d, d, 4 * d * d, 4 * d * d] * case["layers"]


def _offsets(sizes):
    """Where each tensor starts in the flat buffers, and their length: whole blocks for each."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return starts, at


def _tokens(g, n, vocab):
    """Token ids in order of frequency, the frequency falling as one over the rank."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return ((u * math.log(vocab + 1)).exp().floor().long() - 1).clamp_(0, vocab - 1)


def _scale(x):
    """The power of two of each block by which its largest magnitude comes to lie in (224, 448], 448 being the largest
    e4m3 value."""
    top = x.view(-1, BLOCK).abs().amax(1).float().view(torch.int32)
    return ((((top + 0x1FFFFF) >> 23).clamp(min=9) - 8) << 23).view(torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    state = dict(case)
    if case["op"] == "xent":
        n, d, v, t = case["rows"], case["width"], case["vocab"], TYPES[case["type"]]
        state["x"] = normal(n, d).to(t)                         # normalised hidden states
        state["w"] = normal(v, d, std=2.0 / math.sqrt(d)).to(t)   # logits of a standard deviation of two
        state["targets"] = _tokens(g, n, v)
        gone = torch.rand(n, generator=g, device="cuda") < case["ignored"]
        state["targets"][gone] = -100
        # the gradient of the mean over the rows that count
        state["grad_loss"] = torch.where(gone, 0.0, 1.0 / (~gone).sum().clamp(min=1)).float()
    elif case["op"] == "embed":
        n, d, v, t = case["tokens"], case["width"], case["vocab"], TYPES[case["type"]]
        state["ids"] = _tokens(g, n, v)
        state["pad"] = v - 1
        state["ids"][torch.rand(n, generator=g, device="cuda") < case["pads"]] = v - 1
        state["scale"] = math.sqrt(d)
        if case["grads"]:
            state["grad"] = normal(n, d, std=1.0 / n).to(t)
        else:
            state["table"] = normal(v, d, std=0.02).to(t)
    else:
        sizes = _sizes(case)
        starts, total = _offsets(sizes)
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for at, n in zip(starts, sizes):
            inside[at:at + n] = True
        param = torch.where(inside, normal(total, std=0.02), 0.0)
        grad = torch.where(inside, normal(total, std=1e-3), 0.0).to(TYPES[case["type"]])
        m = torch.where(inside, normal(total, std=3e-4), 0.0)
        v = torch.where(inside, normal(total, std=2e-4).abs_().add_(9e-4).square_(), 0.0)
        state.update(param=param, grad=grad, t=AT_STEP)
        # vectors are not decayed
        decay = [DECAY if i == 0 or (i >= 2 and (i - 2) % 5 in (1, 3, 4)) else 0.0 for i in range(len(sizes))]
        blocks = [(n + BLOCK - 1) // BLOCK for n in sizes]
        state["decay"] = torch.tensor(decay, device="cuda").repeat_interleave(torch.tensor(blocks, device="cuda"))
        if case["bits"] == 32:
            state.update(m=m, v=v)
        else:
            for name, x in (("m", m), ("v", v)):
                scale = _scale(x)
                state[name] = (x.view(-1, BLOCK) / scale[:, None]).reshape(-1).to(torch.float8_e4m3fn)
                state[name + "_scale"] = scale
        if case["copy"]:
            state["weights"] = param.to(TYPES[case["type"]])
        if own:
            from paper_2605_17879_b200 import operators
            views = lambda flat: [flat[at:at + n] for at, n in zip(starts, sizes)]  # noqa: E731
            kept = {k: state[k] for k in ("m", "v", "m_scale", "v_scale") if k in state}
            state["opt"] = operators.AdamW(views(param), views(grad), betas=(BETA1, BETA2), eps=EPS, weight_decay=decay,
                                           state_bits=case["bits"], copies=views(state["weights"]) if case["copy"] else None,
                                           state=kept, step=AT_STEP, seed=SEED)
    return state


def run(state):
    return {"xent": _xent, "embed": _embed, "adamw": _adamw}[state["op"]](state)


def _xent(s):
    if own:
        from paper_2605_17879_b200 import operators
        out = operators.linear_xent(s["x"], s["w"], s["targets"])
        if not s["grads"]:
            return {"loss": out["loss"], "lse": out["lse"]}
        back = operators.linear_xent_grad(s["x"], s["w"], s["targets"], out["lse"], s["grad_loss"])
        return {"loss": out["loss"], "lse": out["lse"], "dx": back["dx"], "dw": back["dw"]}
    x, w = s["x"].float(), s["w"].float()
    counts = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    z = x @ w.T
    top = z.amax(1, keepdim=True)
    picked = z.gather(1, at)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    loss = torch.where(counts[:, None], lse - picked, 0.0)
    out = {"loss": loss[:, 0], "lse": torch.where(counts, lse[:, 0], 0.0)}     # rows that are ignored have neither
    if s["grads"]:
        p = (z - lse).exp()
        p.scatter_add_(1, at, torch.full_like(picked, -1.0))
        p *= (s["grad_loss"] * counts)[:, None]
        out["dx"] = (p @ w).to(s["x"].dtype)
        out["dw"] = (p.T @ x).to(s["w"].dtype)
    return out


def _embed(s):
    if own:
        from paper_2605_17879_b200 import operators
        if not s["grads"]:
            return operators.embed(s["ids"], s["table"], scale=s["scale"])["out"]
        return operators.embed_grad(s["grad"], s["ids"], s["vocab"], scale=s["scale"], padding_idx=s["pad"])["dtable"]
    if not s["grads"]:
        return (s["table"][s["ids"]].float() * s["scale"]).to(s["table"].dtype)
    g = s["grad"].float() * (s["ids"] != s["pad"])[:, None]
    total = torch.zeros(s["vocab"], s["width"], device=g.device).index_add_(0, s["ids"], g)
    return (total * s["scale"]).to(s["grad"].dtype)


def _dither(n, t, device):
    """16 + 16 dithering bits of every position, from the step's number and the seed."""
    low, key = 0xFFFFFFFF, (SEED + t * 0x9E3779B9) & 0xFFFFFFFF
    i = torch.arange(n, device=device)
    h = (((i & low) + (i >> 32) * 0x85EBCA6B) & low) ^ key
    h = (h * 0x9E3779B1) & low
    h = h ^ (h >> 15)
    h = (h * 0x85EBCA77) & low
    h = h ^ (h >> 13)
    return (h & 0xFFFF).int(), (h >> 16).int()


def _to_8_bits(x, scale, bits, least):
    """x, in blocks with a scale each, as e4m3 values: dithered by `bits`, so that the mean is x; nonzero values are
    held as one smallest step at least where `least` says so."""
    y = (x.abs().view(-1, BLOCK) / scale[:, None]).view(-1)
    fine = ((y.view(torch.int32) + (bits << 4)) & ~0xFFFFF).view(torch.float32)
    steps = (y * 512 + bits.float() * 2.0 ** -16).floor()
    if least:
        steps = torch.where(y > 0, steps.clamp(min=1.0), steps)
    y = torch.where(y < 2.0 ** -6, steps / 512, fine)
    return torch.copysign(y, x).to(torch.float8_e4m3fn)


def _adamw(s):
    names = [k for k in ("param", "m", "v", "m_scale", "v_scale", "weights") if k in s]
    if own:
        s["opt"].step(LR)
        return {k: s[k] for k in names}
    s["t"] += 1
    c1, c2 = 1 - BETA1 ** s["t"], 1 - BETA2 ** s["t"]
    g, p = s["grad"].float(), s["param"]
    m, v = s["m"], s["v"]
    if s["bits"] == 8:
        m, v = ((x.float().view(-1, BLOCK) * scale[:, None]).view(-1) for x, scale in ((m, s["m_scale"]), (v, s["v_scale"])))
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    kept = (p.view(-1, BLOCK) * (1 - LR * s["decay"])[:, None]).view(-1)
    p.copy_(kept - (LR / c1) * (m / (v.sqrt() / math.sqrt(c2) + EPS)))
    if s["bits"] == 8:
        low, high = _dither(p.numel(), s["t"], p.device)
        for name, x, bits in (("m", m, low), ("v", v, high)):
            s[name + "_scale"].copy_(_scale(x))
            s[name].copy_(_to_8_bits(x, s[name + "_scale"], bits, name == "v"))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if "weights" in s:
        s["weights"].copy_(p)
    return {k: s[k] for k in names}


def _distinct(n, vocab):
    """Expected number of different tokens among n."""
    r = torch.arange(1, vocab + 1, dtype=torch.float64)
    p = torch.log1p(1 / r) / math.log(vocab + 1)
    return float((1 - (1 - p) ** n).sum())


def work(case):
    if case["op"] == "xent":
        n, d, v, b = case["rows"], case["width"], case["vocab"], BYTES[case["type"]]
        once = (n + v) * d * b
        product = 2.0 * n * (1 - case["ignored"]) * v * d      # rows that are ignored need none
        if not case["grads"]:
            return {"bytes": once + n * 16, "flops": product}
        return {"bytes": 2 * once + n * 20, "flops": 3 * product}
    if case["op"] == "embed":
        n, d, v, b = case["tokens"], case["width"], case["vocab"], BYTES[case["type"]]
        if not case["grads"]:
            return {"bytes": n * 8 + (_distinct(n, v) + n) * d * b, "flops": n * d}
        return {"bytes": n * 8 + (n * (1 - case["pads"]) + v) * d * b, "flops": n * (1 - case["pads"]) * d}
    n = sum(_sizes(case))
    states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    each = 8 + BYTES[case["type"]] + states + (BYTES[case["type"]] if case["copy"] else 0)
    return {"bytes": n * each, "flops": 15 * n}


def exact(case, seed):
    """The definitions, in 64 bits."""
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if case["op"] == "xent":
        x, w = s["x"].double(), s["w"].double()
        logp = torch.mm(x, w.t())
        lse = torch.logsumexp(logp, 1)
        logp -= lse[:, None]
        keep = (s["targets"] != -100).double()
        row = torch.arange(len(x), device="cuda")
        at = torch.where(s["targets"] == -100, 0, s["targets"])
        out = {"loss": -logp[row, at] * keep, "lse": lse * keep}
        if case["grads"]:
            q = logp.exp_()
            q[row, at] -= 1.0
            q *= (s["grad_loss"].double() * keep)[:, None]
            out["dx"] = torch.mm(q, w)
            out["dw"] = torch.mm(q.t(), x)
        return out
    if case["op"] == "embed":
        if not case["grads"]:
            return torch.index_select(s["table"], 0, s["ids"]).double() * s["scale"]
        used = s["ids"] != s["pad"]
        total = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
        total.index_put_((s["ids"][used],), s["grad"][used].double() * s["scale"], accumulate=True)
        return total
    t = AT_STEP + 1
    g, p, m, v = s["grad"].double(), s["param"].double(), s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        m *= s["m_scale"].double().repeat_interleave(BLOCK)
        v *= s["v_scale"].double().repeat_interleave(BLOCK)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g ** 2, v, BETA2)
    p = p - LR * s["decay"].double().repeat_interleave(BLOCK) * p
    p = p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    out = {"param": p, "m": m, "v": v, "weights": p if case["copy"] else None}
    if case["bits"] == 8:       # which of two neighbouring 8-bit values is held goes by the dithering bits
        out.update(m=None, v=None, m_scale=_scale(m).double(), v_scale=_scale(v).double())
    return out
