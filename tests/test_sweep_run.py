"""What the node sweep's command makes of the ranks' results, without a GPU: loads and qualification are stand-ins."""
import math
import os
import socket

import pytest
import torch
import torch.multiprocessing as mp

from paper_2605_17879_b200 import sweep_run


def passes(rows, nodes, per):
    """In place of guard.sweep_qualify: a GPU fails where its first metric's median is below 50."""
    med = rows.median(1).values
    ok = med[:, 0] >= 50
    assert nodes * per == len(rows) and rows.isfinite().all()
    return {"gpu_med": med, "fail_mask": (~ok).int(), "gpu_pass": ok.byte()}


def results(gpus, reps=3):
    return torch.full((gpus, reps, 4), 100.0), torch.arange(float(reps)).repeat(gpus, 1)


def test_agreement_takes_whole_rows_and_a_strict_majority():
    a, b, c = [1.0, 2.0], [1.0, 3.0], [0.5, 2.0]
    t = lambda *rows: torch.tensor(rows)    # noqa: E731
    assert sweep_run.agreement(t(a)) == [True]
    assert sweep_run.agreement(t(a, a)) == [True, True]
    assert sweep_run.agreement(t(a, b)) == [None, None]
    assert sweep_run.agreement(t(a, b, a)) == [True, False, True]
    assert sweep_run.agreement(t(a, b, c)) == [None] * 3          # (elementwise, [1, 2] would be the commonest)
    assert sweep_run.agreement(t(a, a, b, b)) == [None] * 4
    nan = [math.nan, 1.0]
    assert sweep_run.agreement(t(nan, nan, a)) == [True, True, False]      # bit for bit
    assert sweep_run.agreement(t([0.0], [-0.0], [0.0])) == [True, False, True]
    assert sweep_run.agreement(torch.empty(0, 3)) == []


def test_verdict():
    rows, losses = results(4)
    got = sweep_run.verdict(rows, losses, [False] * 4, 2, passes)
    assert got["gpu_pass"] == [1] * 4 and got["node_pass"] == [1, 1] and got["same_results"] == [True] * 4 and got["last_loss"] == 2.0
    assert got["medians"][3] == dict.fromkeys(sweep_run.METRICS, 100.0) and got["load_failed"] == [False] * 4
    slow = rows.clone()
    slow[1] = 10
    got = sweep_run.verdict(slow, losses, [False] * 4, 2, passes)
    assert got["gpu_pass"] == [1, 0, 1, 1] and got["node_pass"] == [0, 1] and got["fail_mask"] == [0, 1, 0, 0]
    wrong = losses.clone()
    wrong[2, 0] += 1                                               # fast, but wrong
    got = sweep_run.verdict(rows, wrong, [False] * 4, 2, passes)
    assert got["gpu_pass"] == [1, 1, 0, 1] and got["node_pass"] == [1, 0] and got["same_results"] == [True, True, False, True]
    broken = rows.clone()
    broken[0] = math.nan                                           # its load failed: the others are qualified without it
    got = sweep_run.verdict(broken, losses, [True, False, False, False], 2, passes)
    assert got["gpu_pass"] == [0, 1, 1, 1] and got["node_pass"] == [0, 1] and got["medians"][0] is None and got["same_results"][0] is None
    got = sweep_run.verdict(broken, losses, [True] * 4, 4, passes)
    assert got["gpu_pass"] == [0] * 4 and got["node_pass"] == [0] and got["last_loss"] is None


class Load:
    def __init__(self, rank, how):
        if how == "cannot start":
            raise RuntimeError("no memory")
        self.rank, self.how = rank, how

    def measure(self, reps):
        if self.how == "runs out":
            from paper_2605_17879_b200.guard import GuardError
            raise GuardError(-5, "a wait ran out")
        return {"rows": torch.full((reps, 4), 100.0 + self.rank), "loss": torch.arange(float(reps)) + (self.how == "wrong")}


def _rank(rank, port, hows, q):
    os.environ.update(RANK=str(rank), LOCAL_RANK=str(rank), WORLD_SIZE=str(len(hows)), MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    from paper_2605_17879_b200 import dist as gd
    gd.init("gloo")
    q.put((rank, *sweep_run.sweep(lambda: Load(rank, hows[rank]), 3, len(hows), passes)))
    gd.barrier()
    gd.finish()


@pytest.mark.parametrize("hows,reporter,gpu_pass,codes", [
    (["", "", ""], 0, [1, 1, 1], [0, 0, 0]), (["", "runs out", ""], 0, [1, 0, 1], [0, 1, 0]),
    (["cannot start", "", "runs out"], 1, [0, 1, 0], [1, 0, 1]), (["", "", "wrong"], 0, [1, 1, 0], [1, 0, 0]),
    (["runs out", "cannot start"], 0, [0, 0], [1, 1]), (["", "wrong"], 0, [1, 1], [1, 0])])
def test_a_rank_whose_load_fails_is_reported(hows, reporter, gpu_pass, codes):
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    procs = [ctx.Process(target=_rank, args=(r, port, hows, q)) for r in range(len(hows))]
    for p in procs:
        p.start()
    res = {r: (report, code) for r, report, code in (q.get(timeout=120) for _ in procs)}
    for p in procs:
        p.join(timeout=60)
        assert p.exitcode == 0
    assert [res[r][1] for r in range(len(hows))] == codes
    assert [r for r in res if res[r][0] is not None] == [reporter]
    report = res[reporter][0]
    assert report["gpu_pass"] == gpu_pass and report["load_failed"] == [h in ("runs out", "cannot start") for h in hows]


def test_one_process_needs_no_group():
    report, code = sweep_run.sweep(lambda: Load(0, ""), 2, 1, passes)
    assert code == 0 and report["gpu_pass"] == [1] and report["same_results"] == [True]
    report, code = sweep_run.sweep(lambda: Load(0, "runs out"), 2, 1, passes)
    assert code == 1 and report["gpu_pass"] == [0] and report["load_failed"] == [True]
