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


@pytest.mark.parametrize("limit", [1, 300, 3000, 10000, 30000, 90000])
@pytest.mark.parametrize("n,d,v", [(300, 256, 3000), (600, 2048, 20000), (60, 512, 8192)])
def test_a_wait_that_runs_out_is_reported_and_later_calls_work(ops, n, d, v, limit):
    """With a limit of some clock cycles waits inside the products run out, at the first stage or in the middle of the work,
    while copies and products are in flight.  The kernels let those land and return; a call that reports nothing is right."""
    g = gen(n)
    x = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * (2 / d ** 0.5)).bfloat16()
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    one = torch.full((1,), 1.0 / n, device="cuda")
    want = ops.linear_xent(x, w, t)
    back = ops.linear_xent_grad(x, w, t, want["lse"], one)
    ops.sync_status()

    def status():
        return torch.zeros(1, dtype=torch.uint32, device="cuda")
    ran_out = 0
    for _ in range(5):
        out = {"loss": torch.empty(n, device="cuda"), "lse": torch.empty(n, device="cuda"), "status": status()}
        grads = {"dx": torch.empty_like(x), "dw": torch.empty_like(w), "status": status()}
        ops.debug_set_wait_limit(limit)
        try:
            ops.linear_xent(x, w, t, out=out)
            ops.linear_xent_grad(x, w, t, want["lse"], one, out=grads)
        finally:
            ops.debug_set_wait_limit(0)
        torch.cuda.synchronize()
        for got, ref in ((out, want), (grads, back)):
            bits = int(got["status"].item())
            assert bits in (0, ops.STATUS_TIMEOUT)
            ran_out += bits != 0
            if not bits:
                assert all(torch.equal(got[k], ref[k]) for k in ref)
        again = ops.linear_xent(x, w, t)
        again_back = ops.linear_xent_grad(x, w, t, again["lse"], one)
        ops.sync_status()
        assert torch.equal(again["loss"], want["loss"]) and torch.equal(again_back["dx"], back["dx"]) and torch.equal(again_back["dw"], back["dw"])
    if limit == 1:
        assert ran_out == 10


def test_adamw_refuses_scalars_off_their_alignment(ops):
    p, grad = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    opt = ops.AdamW([p], [grad])
    two = torch.ones(2, device="cuda")
    step, stream = ops.lib().guard_adamw_step, torch.cuda.current_stream().cuda_stream
    assert step(opt._h, 0.0, two.data_ptr() + 2, None, stream) == -1
    assert step(opt._h, 1e-3, None, two.data_ptr() + 1, stream) == -1
    assert opt.steps() == 0 and (p == 1).all()
    assert step(opt._h, 0.0, two.data_ptr() + 4, two.data_ptr(), stream) == 0
    assert opt.steps() == 1


def test_adamw_is_not_made_or_asked_inside_a_capture(ops):
    """Making an optimiser copies its table from host memory, asking for its steps copies to it: neither address lives when a
    graph is replayed.  The capture itself goes on."""
    p, grad = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    opt = ops.AdamW([p], [grad])
    opt.step(1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ops.GuardError):
            ops.AdamW([torch.ones(8, device="cuda")], [torch.ones(8, device="cuda")])
        with pytest.raises(ops.GuardError):
            opt.steps()
        opt.step(1e-3)
    assert opt.steps() == 1
    graph.replay()
    graph.replay()
    assert opt.steps() == 3


@pytest.mark.parametrize("n", [6, 9000])
@pytest.mark.parametrize("token", [-1, -2 ** 63, 2 ** 63 - 1, 4])
def test_every_token_outside_the_table_is_an_error(ops, n, token):
    grad = torch.ones(n, 8, device="cuda")
    ids = torch.arange(n, device="cuda") % 4
    ids[5] = token
    for padding in (-1, 2):
        out = {"dtable": torch.empty(4, 8, device="cuda"), "status": torch.zeros(1, dtype=torch.uint32, device="cuda")}
        ops.embed_grad(grad, ids, 4, padding_idx=padding, out=out)
        assert int(out["status"].item()) == ops.STATUS_INDEX
        want = [float(((ids == v) & (v != padding)).sum()) for v in range(4)]
        assert out["dtable"][:, 0].tolist() == want


GIL_STUB = r"""
#include <stddef.h>
extern int PyGILState_Check(void);
static int held;
int stub_held(void) { return held; }
#define STUB(name) int name() { held += PyGILState_Check(); return 0; }
STUB(guard_embed) STUB(guard_embed_grad) STUB(guard_linear_xent) STUB(guard_linear_xent_grad)
"""
GIL_CALLS = r"""
import ctypes, sys, torch
from paper_2605_17879_b200 import operators as ops
held = ctypes.CDLL(sys.argv[1]).stub_held
x = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
t = torch.zeros(4, dtype=torch.int64, device="cuda")
f = torch.zeros(4, device="cuda")
got = []
for call in (lambda: ops.embed(t, x), lambda: ops.embed_grad(x, t, 4), lambda: ops.linear_xent(x, x, t), lambda: ops.linear_xent_grad(x, x, t, f, f)):
    before = held()
    call()
    got.append(held() - before)
print("held", got)
"""


def test_native_calls_release_the_interpreter_lock(tmp_path):
    """The library's entries are replaced by ones that say whether the calling thread holds the lock."""
    import os
    import subprocess
    import sys
    (tmp_path / "stub.c").write_text(GIL_STUB)
    so = str(tmp_path / "stub.so")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", so, str(tmp_path / "stub.c")])
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", GIL_CALLS, so], cwd=root, env=dict(os.environ, LD_PRELOAD=so, PYTHONPATH=root), capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "held [0, 0, 0, 0]" in r.stdout, r.stdout


def test_autograd_notices_what_the_operators_overwrite(ops):
    """A tensor that a backward pass still needs and that a call has written into since: torch refuses it, as it does after its
    own in-place operations."""
    g = gen(3)
    x, w = torch.randn(4, 8, generator=g, device="cuda").bfloat16(), torch.randn(16, 8, generator=g, device="cuda").bfloat16()
    t = torch.tensor([1, 5, 5, 2], device="cuda")
    first = ops.linear_xent(x, w, t)
    one = torch.ones(1, device="cuda")

    def refused(buffer, call):
        leaf = torch.ones((), dtype=buffer.dtype, device="cuda", requires_grad=True)
        y = (buffer * leaf).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    out = torch.empty(4, 8, dtype=torch.bfloat16, device="cuda")
    refused(out, lambda: ops.embed(t, w, out={"out": out}))
    table = torch.zeros(16, 8, dtype=torch.bfloat16, device="cuda")
    refused(table, lambda: ops.embed_grad(x, t, 16, accumulate=True, out={"dtable": table}))
    for name in ("loss", "lse"):
        refused(first[name], lambda: ops.linear_xent(x, w, t, out=first))
    back = ops.linear_xent_grad(x, w, t, first["lse"], one)
    for name in ("dx", "dw"):
        refused(back[name], lambda: ops.linear_xent_grad(x, w, t, first["lse"], one, out=back))
    p, copy = torch.ones(300, device="cuda"), torch.ones(300, device="cuda").bfloat16()
    opt = ops.AdamW([p], [torch.ones(300, device="cuda")], copies=[copy])
    for buffer in (p, copy, opt.state["m"]):
        refused(buffer, lambda: opt.step(1e-3))
    # inputs are not written, and what inference mode made has no versions
    leaf = torch.ones((), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = (x * leaf).sum()
    ops.linear_xent_grad(x, w, t, first["lse"], one)
    y.backward()
    with torch.inference_mode():
        out = torch.empty(4, 8, dtype=torch.bfloat16, device="cuda")
        q = torch.ones(300, device="cuda")
        ops.embed(t, w, out={"out": out})
        opt = ops.AdamW([q], [torch.ones(300, device="cuda")])
    ops.embed(t, w, out={"out": out})
    opt.step(1e-3)
    assert torch.equal(out, w[t]) and opt.steps() == 1


def test_adamw_memory_outlives_a_step_on_another_stream(ops):
    """An optimiser that is dropped while a step of it still runs elsewhere: what it had allocated is not handed out before that."""
    p, grad = torch.ones(100000, device="cuda"), torch.ones(100000, device="cuda")
    opt = ops.AdamW([p], [grad])
    opt.step(1e-3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)           # a fifth of a second
        opt.step(1e-3)
    mine = {t.data_ptr() for t in (opt._ws, *opt.state.values())}
    sizes = [t.untyped_storage().nbytes() for t in (opt._ws, *opt.state.values())]
    running = side.record_event()
    del opt
    again = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    assert not running.query()                    # (the step is still to come)
    assert not mine & {t.data_ptr() for t in again}
    side.synchronize()


def test_adamw_steps_elsewhere_behind_its_making(ops):
    """The table of tensors and the states are made in the order of the constructor's stream; a step on another stream waits
    for them by itself."""
    want = torch.ones(5000, device="cuda")
    grad = torch.full((5000,), 0.5, device="cuda")
    opt = ops.AdamW([want], [grad])
    opt.step(1e-2)
    p = torch.ones(5000, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)               # a tenth of a second
    opt = ops.AdamW([p], [grad])
    with torch.cuda.stream(side):
        opt.step(1e-2)
    side.synchronize()
    assert torch.equal(p, want) and opt.steps() == 1
    # a capture brings its own stream, and may not wait for work outside it: everything has been waited for before
    opt = ops.AdamW([p], [grad])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(1e-2)
    graph.replay()
    assert opt.steps() == 1


def test_threads_call_at_the_same_time(ops):
    """Native calls run without the interpreter lock: threads on streams of their own get their own results and their own
    errors."""
    from concurrent.futures import ThreadPoolExecutor
    g = gen(21)
    shapes = [(200, 64, 500), (60, 512, 3000), (300, 1032, 700), (1000, 72, 257)]
    jobs = []
    for n, d, v in shapes:
        x = torch.randn(n, d, generator=g, device="cuda").bfloat16()
        w = (torch.randn(v, d, generator=g, device="cuda") * (2 / d ** 0.5)).bfloat16()
        t = torch.randint(0, v, (n,), generator=g, device="cuda")
        jobs.append((x, w, t, torch.full((1,), 1.0 / n, device="cuda")))

    def run(x, w, t, one):
        out = ops.linear_xent(x, w, t)
        back = ops.linear_xent_grad(x, w, t, out["lse"], one)
        rows = ops.embed(t, w)["out"]
        return [out["loss"], back["dx"], back["dw"], rows, ops.embed_grad(rows, t, len(w))["dtable"]]
    want = [run(*job) for job in jobs]
    torch.cuda.synchronize()

    def worker(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = run(*jobs[k])
                with pytest.raises(ops.GuardError, match="width a multiple of 8" if k % 2 else "padding_idx"):
                    if k % 2:
                        ops.linear_xent(jobs[k][0][:, :12].contiguous(), jobs[k][1][:, :12].contiguous(), jobs[k][2])
                    else:
                        ops.embed_grad(got[3], jobs[k][2], len(jobs[k][1]), padding_idx=-7)
                assert all(torch.equal(a, b) for a, b in zip(got, want[k]))
        return True
    with ThreadPoolExecutor(len(jobs)) as pool:
        assert all(pool.map(worker, range(len(jobs))))
    ops.sync_status()


def test_outputs_have_no_history(ops):
    """Gradients are calls of their own: nothing is recorded, also where inputs require gradients."""
    g = gen(22)
    w = torch.randn(16, 8, generator=g, device="cuda").bfloat16().requires_grad_()
    x = torch.randn(4, 8, generator=g, device="cuda").bfloat16().requires_grad_()
    t = torch.tensor([1, 5, 5, 2], device="cuda")
    out = ops.linear_xent(x, w, t)
    back = ops.linear_xent_grad(x, w, t, out["lse"], torch.ones(1, device="cuda"))
    for y in (*out.values(), *back.values(), *ops.embed(t, w).values(), *ops.embed_grad(x, t, 16).values()):
        assert not y.requires_grad and y.grad_fn is None
