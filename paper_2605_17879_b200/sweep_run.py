"""The measuring half of the node sweep: a load that makes the results guard.sweep_qualify scores.

Section 5.2's sweep runs benchmarks on every GPU and Section 5.4's rule judges them against the fleet.  The load here is
a training step of the smallest language model that has one: the rows of the next tokens are predicted from the embedding
of the current ones with the same table (tied weights).  A step is

    x = sqrt(width) * weights[tokens];  loss = cross entropy of x weights^T;  gradients;  AdamW of the one table

with the library's own operators (operators.py).  Its parts load what a job's step loads and a product or a copy alone does
not: irregular reads of the table (embed), the tensor cores under the power limit (loss and gradients), a sort and sums over
frequent tokens (embed_grad), and a stream over all of parameters and states (AdamW).  Every part is deterministic, so GPUs
that start from the same seed must report the same losses, bit for bit; one that does not computes wrong results and fails.
So does one whose load raises an error; the others are qualified without it.  The command prints the verdict as one line of JSON
and returns 1 where a load failed or results disagree.

    python -m paper_2605_17879_b200.sweep_run                                         one GPU
    torchrun --standalone --local-addr 127.0.0.1 --nproc-per-node 8 -m paper_2605_17879_b200.sweep_run     a node
"""
from __future__ import annotations

import argparse
import json
import math
import sys
from collections import Counter
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import dist as gd
from . import guard, operators

# What a repetition measures, and in which direction it is bad (guard.sweep_qualify's `dir`).
METRICS = ("loss_tflops", "update_gbs", "embed_gbs", "step_ms")
DIR = (-1, -1, -1, 1)


class SweepStep:
    """The load of one GPU: model, states and buffers, made from the seed alone."""

    def __init__(self, *, rows: int = 8192, width: int = 2048, vocab: int = 65536, state_bits: int = 32, lr: float = 1e-3,
                 seed: int = 0, device="cuda"):
        if rows < 1 or vocab < 2 or width < 8 or width % 8:
            raise ValueError("need rows >= 1, vocab >= 2 and width a multiple of 8")
        self.rows, self.width, self.vocab, self.lr, self.bits = rows, width, vocab, lr, state_bits
        self.scale = math.sqrt(width)
        dev = self.device = torch.device(device)
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.param = torch.randn(vocab, width, generator=g, device=dev).mul_(1.0 / width)
        self.weights = self.param.bfloat16()
        self.grad = torch.empty_like(self.weights)
        self.opt = operators.AdamW([self.param], [self.grad], betas=(0.9, 0.95), weight_decay=0.1, state_bits=state_bits,
                                   copies=[self.weights], seed=seed)
        # tokens by falling frequency; what follows a token is a fixed choice nine times out of ten
        u = torch.rand(rows, generator=g, device=dev, dtype=torch.float64)
        self.tokens = (((vocab + 1.0) ** u).long() - 1).clamp_(0, vocab - 1)
        follow = torch.randperm(vocab, generator=g, device=dev)[self.tokens]
        other = torch.randint(0, vocab, (rows,), generator=g, device=dev)
        self.targets = torch.where(torch.rand(rows, generator=g, device=dev) < 0.9, follow, other)
        self.mean = torch.full((1,), 1.0 / rows, device=dev)
        self.x = {"out": torch.empty(rows, width, dtype=torch.bfloat16, device=dev)}
        self.loss = {"loss": torch.empty(rows, device=dev), "lse": torch.empty(rows, device=dev)}
        self.back = {"dx": torch.empty(rows, width, dtype=torch.bfloat16, device=dev), "dw": self.grad}
        L = operators.lib()

        def space(n):
            return torch.empty(int(n), dtype=torch.uint8, device=dev)
        self.ws = (space(L.guard_linear_xent_workspace_bytes(rows, width, vocab, 0)), space(L.guard_linear_xent_workspace_bytes(rows, width, vocab, 1)),
                   space(L.guard_embed_grad_workspace_bytes(rows, vocab, width)))

    def step(self, mark=lambda k: None) -> torch.Tensor:
        """One training step; returns the row losses (a buffer that the next step overwrites).  mark(k) is called before
        part k: 0 lookup, 1 loss and gradients, 2 gradient of the lookup, 3 update, and 4 at the end."""
        x, w = self.x["out"], self.weights
        mark(0)
        operators.embed(self.tokens, w, scale=self.scale, out=self.x)
        mark(1)
        operators.linear_xent(x, w, self.targets, workspace=self.ws[0], out=self.loss)
        operators.linear_xent_grad(x, w, self.targets, self.loss["lse"], self.mean, workspace=self.ws[1], out=self.back)
        mark(2)
        operators.embed_grad(self.back["dx"], self.tokens, self.vocab, scale=self.scale, accumulate=True, workspace=self.ws[2],
                             out={"dtable": self.grad})
        mark(3)
        self.opt.step(self.lr)
        mark(4)
        return self.loss["loss"]

    def measure(self, reps: int, warmup: int = 3) -> Dict[str, torch.Tensor]:
        """`rows` [reps, 4] float32: the METRICS of each repetition (one step), timed on the GPU; `loss` [reps] float32: the
        mean loss of each, the same on every healthy GPU."""
        if reps < 1:
            raise ValueError("reps must be at least 1")
        n, d, v = self.rows, self.width, self.vocab
        flops = 8.0 * n * v * d                                     # logits, logits again, both gradients
        update = v * d * (8 + 2 + 2 + (16 if self.bits == 32 else 4 + 16 / operators.BLOCK))
        moved = n * d * 2.0 * 5                                     # lookup: read, written; gradient: read, rows read and written
        out = torch.empty(reps, len(METRICS))
        loss = torch.empty(reps, device=self.device)
        with torch.cuda.device(self.device):
            for _ in range(warmup):
                self.step()
            events = [[torch.cuda.Event(enable_timing=True) for _ in range(5)] for _ in range(reps)]
            for r in range(reps):
                each = self.step(lambda k: events[r][k].record())
                torch.mean(each, 0, out=loss[r])
            operators.sync_status(self.device)
            torch.cuda.synchronize(self.device)
            for r, e in enumerate(events):
                lookup, product, back, opt = (e[k].elapsed_time(e[k + 1]) for k in range(4))      # milliseconds
                out[r] = torch.tensor([flops / product / 1e9, update / opt / 1e6, moved / (lookup + back) / 1e6, e[0].elapsed_time(e[4])])
        return {"rows": out.to(self.device), "loss": loss}


def qualify(rows: torch.Tensor, nodes: int, gpus_per_node: int, **kw):
    """guard.sweep_qualify of measured rows [gpus, reps, 4], with this load's directions."""
    return guard.sweep_qualify(rows.contiguous(), nodes, gpus_per_node, dir=DIR, **kw)


def agreement(losses: torch.Tensor) -> List[Optional[bool]]:
    """Which GPUs computed what most of them did: losses [gpus, reps], compared whole and bit for bit.  True and False where a
    strict majority agrees, None for all where there is none."""
    rows = [tuple(r) for r in losses.contiguous().view(torch.int32).tolist()]
    common, count = Counter(rows).most_common(1)[0] if rows else ((), 0)
    return [r == common for r in rows] if 2 * count > len(rows) else [None] * len(rows)


def verdict(rows: torch.Tensor, losses: torch.Tensor, failed: Sequence[bool], gpus_per_node: int, qualifier=qualify) -> Dict[str, object]:
    """What the fleet's results say.  rows [gpus, reps, 4], losses [gpus, reps], failed: GPUs whose load raised an error, whose
    results say nothing.  Those fail; the others are qualified against one another, and fail too where they computed other
    losses than the majority.  A node passes when all its GPUs pass."""
    gpus, reps = losses.shape
    good = [g for g in range(gpus) if not failed[g]]
    medians, fail_mask, same = [None] * gpus, [None] * gpus, [None] * gpus
    gpu_pass = [0] * gpus
    if good:
        out = qualifier(rows[good], len(good), 1)
        equal = agreement(losses[good])
        for k, g in enumerate(good):
            medians[g] = dict(zip(METRICS, [round(float(x), 3) for x in out["gpu_med"][k]]))
            fail_mask[g], same[g] = int(out["fail_mask"][k]), equal[k]
            gpu_pass[g] = int(bool(out["gpu_pass"][k]) and equal[k] is not False)
    return {"metrics": METRICS, "gpus": gpus, "reps": reps, "medians": medians, "gpu_pass": gpu_pass,
            "node_pass": [min(gpu_pass[n:n + gpus_per_node]) for n in range(0, gpus, gpus_per_node)], "fail_mask": fail_mask,
            "same_results": same, "load_failed": [bool(f) for f in failed], "last_loss": float(losses[good[0], -1]) if good else None}


def sweep(make, reps: int, gpus_per_node: int, qualifier=qualify) -> Tuple[Optional[Dict[str, object]], int]:
    """Runs the load make() on this rank and collects every rank's results on the host, where a GPU that failed its load can
    still report.  Returns the verdict on the first rank whose load ran (None on the others), and 1 where this rank's load
    failed or the results that were collected disagree."""
    rank, _, _ = gd.env_world()
    rows, loss, load = torch.full((reps, len(METRICS)), math.nan), torch.full((reps,), math.nan), None
    error = None
    try:
        load = make()
    except (guard.GuardError, RuntimeError) as e:
        error = e
    gd.barrier()                    # all of them start together
    try:
        if load is not None:
            got = load.measure(reps)
            rows, loss = got["rows"].cpu(), got["loss"].cpu()
    except (guard.GuardError, RuntimeError) as e:
        error = e
    if error is not None:
        print("rank %d: the load failed: %s" % (rank, error), file=sys.stderr, flush=True)
    failed = gd.gather(torch.tensor([error is not None])).flatten().tolist()
    S, losses = gd.gather(rows), gd.gather(loss)
    if rank != (failed.index(False) if False in failed else 0):
        return None, int(error is not None)
    report = verdict(S, losses, failed, gpus_per_node, qualifier)
    agree = all(report["same_results"][g] is True for g in range(len(failed)) if not failed[g])
    return report, int(error is not None or not agree)


def main(argv: Optional[list] = None) -> int:
    ap = argparse.ArgumentParser(description="Runs the sweep's load on every rank's GPU and qualifies the GPUs against one another.")
    ap.add_argument("--reps", type=int, default=20)
    ap.add_argument("--rows", type=int, default=8192)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--vocab", type=int, default=65536)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--gpus-per-node", type=int, default=0, help="ranks of a node (default: all)")
    args = ap.parse_args(argv)
    if not torch.cuda.is_available():
        raise SystemExit("sweep_run needs a CUDA device (there is no CPU fallback)")
    if args.reps < 1:
        raise SystemExit("--reps must be at least 1")
    # (the ranks exchange rows of results only, and those on the host)
    rank, local_rank, world = gd.init("gloo")
    per_node = args.gpus_per_node or world
    if world % per_node:
        raise SystemExit("the number of ranks must be a multiple of --gpus-per-node")
    device = torch.device("cuda", local_rank)
    torch.cuda.set_device(device)
    report, code = sweep(lambda: SweepStep(rows=args.rows, width=args.width, vocab=args.vocab, state_bits=args.state_bits, device=device),
                         args.reps, per_node, lambda S, nodes, per: {k: v.cpu() for k, v in qualify(S.to(device), nodes, per).items()})
    if report is not None:
        print(json.dumps(report), flush=True)
    gd.barrier()                    # (a launcher ends the other ranks when one returns an error)
    gd.finish()
    return code


if __name__ == "__main__":
    sys.exit(main())
