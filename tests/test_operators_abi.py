"""Refusals of the training-step operators, which need no GPU: every call below fails before any CUDA work."""
import ctypes as C

import pytest
import torch

from paper_2605_17879_b200 import build as gbuild

P = 256 * 4096          # an address that is never dereferenced
Q = P + (1 << 40)
WS = Q + (1 << 40)


@pytest.fixture(scope="module")
def L():
    gbuild.build_library()
    from paper_2605_17879_b200 import operators
    return operators.lib()


def text(L):
    return L.guard_last_error(None).decode()


def test_embed_refusals(L):
    def call(tokens=P, bits=64, n=4, table=Q, rows=8, width=16, stride=16, dtype=1, out=WS):
        return L.guard_embed(tokens, bits, n, table, rows, width, stride, dtype, 1.0, out, None, None)
    assert call(n=0) == 0 and call(n=0, tokens=None, out=None) == 0
    for bad in (dict(bits=16), dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(rows=-1), dict(width=0), dict(stride=15), dict(width=1 << 25, stride=1 << 25),
                dict(tokens=None), dict(table=None), dict(out=None), dict(tokens=P + 4), dict(table=Q + 1), dict(out=WS + 1), dict(n=1 << 60),
                dict(out=Q + 32), dict(out=P)):
        assert call(**bad) == -1, bad
        assert text(L)


def test_embed_grad_refusals(L):
    need = L.guard_embed_grad_workspace_bytes(100, 50, 16)
    assert need > 0 and need % 256 == 0
    for bad in ((-1, 50, 16), (1 << 31, 50, 16), (100, -1, 16), (100, (1 << 31) - 1, 16), (100, 50, 0)):
        assert L.guard_embed_grad_workspace_bytes(*bad) == 0
    def call(grad=P, stride=16, dtype=1, tokens=P + (1 << 30), bits=64, n=100, rows=50, width=16, pad=-1, acc=0, out=Q, ws=WS, nws=need):
        return L.guard_embed_grad(grad, stride, dtype, tokens, bits, n, rows, width, 1.0, pad, acc, out, ws, nws, None, None)
    assert call(rows=0) == 0 and call(n=0, acc=1) == 0
    for bad in (dict(bits=8), dict(dtype=7), dict(n=-1), dict(stride=8), dict(width=0), dict(pad=-2), dict(pad=50), dict(grad=None), dict(tokens=None),
                dict(out=None), dict(grad=P + 1), dict(out=P), dict(out=P + (1 << 30)), dict(out=WS)):
        assert call(**bad) == -1, bad
    for bad in (dict(ws=None), dict(ws=WS + 16), dict(nws=need - 1)):
        assert call(**bad) == -2, bad


def test_cross_entropy_refusals(L):
    need = {g: L.guard_linear_xent_workspace_bytes(300, 64, 1000, g) for g in (0, 1)}
    assert need[0] > 0 and need[1] > need[0] and need[0] % 256 == 0 and need[1] % 256 == 0
    for bad in ((0, 64, 1000), (300, 0, 1000), (300, 60, 1000), (300, 64, 0), ((1 << 26) + 1, 64, 1000), (300, 64, 1 << 31), (1 << 30, 64, 1 << 30), (300, 1 << 25, 1000)):
        assert L.guard_linear_xent_workspace_bytes(*bad, 0) == 0, bad
    big = 1 << 40
    def forward(x=P, xs=64, w=Q, wst=64, n=300, d=64, v=1000, dtype=1, t=WS, bits=64, loss=WS + big, lse=WS + big + 4096, ws=WS + 2 * big, nws=need[0]):
        return L.guard_linear_xent(x, xs, w, wst, n, d, v, dtype, t, bits, -100, loss, lse, ws, nws, None, None)
    def backward(x=P, xs=64, w=Q, wst=64, n=300, d=64, v=1000, dtype=1, t=WS, bits=64, lse=WS + big, g=WS + big + 4096, gs=1, dx=WS + 2 * big, dw=WS + 3 * big,
                 ws=WS + 4 * big, nws=need[1]):
        return L.guard_linear_xent_grad(x, xs, w, wst, n, d, v, dtype, t, bits, -100, lse, g, gs, dx, dw, ws, nws, None, None)
    assert forward(n=0) == 0 and backward(n=0, dw=None) == 0
    both = (dict(dtype=0), dict(dtype=3), dict(bits=16), dict(xs=56), dict(xs=68), dict(wst=60), dict(wst=0), dict(d=60), dict(n=-1), dict(v=0), dict(x=None), dict(w=None),
            dict(t=None), dict(x=P + 2), dict(w=Q + 8), dict(t=WS + 4))
    for bad in both + (dict(loss=None), dict(lse=None), dict(lse=WS + big + 2), dict(loss=P), dict(lse=WS + big + 100), dict(loss=WS + 8), dict(loss=WS + 2 * big)):
        assert forward(**bad) == -1, bad
        assert text(L)
    for bad in both + (dict(lse=None), dict(g=None), dict(gs=2), dict(dx=None, dw=None), dict(dx=WS + 2 * big + 8), dict(dw=Q), dict(dx=P + 16), dict(dw=WS + 2 * big),
                       dict(dx=WS + 4 * big), dict(dx=WS + big)):
        assert backward(**bad) == -1, bad
    for bad in (dict(ws=None), dict(ws=WS + 2 * big + 64), dict(nws=need[0] - 1)):
        assert forward(**bad) == -2, bad
    assert backward(nws=need[1] - 1) == -2


def test_adamw_refusals(L):
    from paper_2605_17879_b200 import operators as ops
    h = C.c_void_p()
    def call(tensors=((P, Q, None, 1000, 0.1), (P + 4096, Q + 4096, None, 10, 0.0)), n=None, gt=1, ct=1, bits=32, b1=0.9, b2=0.99, eps=1e-8, m=WS,
             v=WS + (1 << 20), ms=None, vs=None, step=0, ws=WS + (1 << 30), nws=1 << 20):
        t = (ops._AdamwTensor * max(1, len(tensors)))(*[ops._AdamwTensor(*x) for x in tensors])
        return L.guard_adamw_create(C.byref(h), t, len(tensors) if n is None else n, gt, ct, bits, b1, b2, eps, m, v, ms, vs, step, 0, ws, nws, None)
    inf = float("inf")
    for bad in (dict(n=0), dict(n=-1), dict(gt=3), dict(ct=-1), dict(bits=16), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(eps=-1.0), dict(eps=0.0), dict(eps=1e300),
                dict(eps=inf), dict(step=-1), dict(m=None), dict(v=WS + 8), dict(bits=8), dict(tensors=((P, Q, None, -1, 0.0),)), dict(tensors=((None, Q, None, 5, 0.0),)),
                dict(tensors=((P, None, None, 5, 0.0),)), dict(tensors=((P + 2, Q, None, 5, 0.0),)), dict(tensors=((P, Q + 1, None, 5, 0.0),)),
                dict(tensors=((P, Q, None, 5, inf),)),
                dict(tensors=((P, Q, None, 1000, 0.0), (P, Q + 4096, None, 10, 0.0))),              # the same parameter twice
                dict(tensors=((P, Q, P + 8, 1000, 0.0),)), dict(tensors=((P, P, None, 1000, 0.0),)),  # copy or gradient inside it
                dict(tensors=((P, Q, Q, 1000, 0.0),)), dict(m=P), dict(v=WS), dict(ws=WS)):
        assert call(**bad) == -1, bad
        assert h.value is None
    for bad in (dict(ws=None), dict(ws=WS + (1 << 30) + 8), dict(nws=300)):
        assert call(**bad) == -2, bad
    t = (ops._AdamwTensor * 3)(ops._AdamwTensor(P, Q, None, 0, 0.0), ops._AdamwTensor(P, Q, None, 257, 0.0), ops._AdamwTensor(P, Q, None, 256, 0.0))
    assert L.guard_adamw_blocks(t, 3) == 3 and L.guard_adamw_blocks(t, 0) == 0 and L.guard_adamw_blocks(None, 1) == -1
    assert L.guard_adamw_step(None, 1e-3, None, None, None) == -1
    assert L.guard_adamw_steps(None, None, None) == -1
    L.guard_adamw_destroy(None)


def test_binding_refusals(L):
    from paper_2605_17879_b200 import operators as ops
    x = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        ops.embed(ids, x)                       # CPU tensors
    with pytest.raises(ValueError):
        ops.embed_grad(x, ids, 4)
    with pytest.raises(ValueError):
        ops.AdamW([x], [x])
    with pytest.raises(ValueError):
        ops.AdamW([], [])
    with pytest.raises(ValueError):
        ops.AdamW([x], [x], state_bits=16)
    with pytest.raises(ValueError):
        ops.linear_xent(x, x, ids)
    with pytest.raises(ValueError):
        ops.linear_xent_grad(x, x, ids, x, x)
    assert ops.AdamW.state_blocks([torch.zeros(0), torch.zeros(257)]) == 2


def test_wait_limit_refusals(L):
    from paper_2605_17879_b200 import operators as ops
    assert L.guard_debug_set_operator_wait_limit(-1) == -1 and text(L)
    with pytest.raises(ops.GuardError):
        ops.debug_set_wait_limit(-5)
    ops.debug_set_wait_limit(0)


def test_scalars_must_be_aligned(L):
    """A float32 or a status word that the kernels access must lie on four bytes."""
    assert L.guard_embed(P, 64, 4, Q, 8, 16, 16, 1, 1.0, WS, WS + (1 << 30) + 2, None) == -1
    assert "status" in text(L)
    assert L.guard_embed_grad(P, 16, 1, P + (1 << 30), 64, 100, 50, 16, 1.0, -1, 0, Q, WS, 1 << 30, P + (1 << 31) + 1, None) == -1
    big = 1 << 40
    assert L.guard_linear_xent(P, 64, Q, 64, 300, 64, 1000, 1, WS, 64, -100, WS + big, WS + big + 4096, WS + 2 * big, 1 << 30, WS + 3 * big + 2, None) == -1
    assert L.guard_linear_xent_grad(P, 64, Q, 64, 300, 64, 1000, 1, WS, 64, -100, WS + big, WS + big + 4096, 1, WS + 2 * big, WS + 3 * big, WS + 4 * big, 1 << 30,
                                    WS + 5 * big + 3, None) == -1
    assert "status" in text(L)


def test_inputs_must_not_lie_in_the_workspace(L):
    need = L.guard_embed_grad_workspace_bytes(100, 50, 16)
    def embed(grad=P, tokens=P + (1 << 30), out=Q, ws=WS):
        return L.guard_embed_grad(grad, 16, 1, tokens, 64, 100, 50, 16, 1.0, -1, 0, out, ws, need, None, None)
    assert embed(grad=WS + 512) == -1 and embed(tokens=WS + need - 8) == -1 and embed(tokens=WS - 8) == -1
    assert "workspace" in text(L)
    big = 1 << 40
    need = {g: L.guard_linear_xent_workspace_bytes(300, 64, 1000, g) for g in (0, 1)}
    def forward(x=P, w=Q, t=WS):
        return L.guard_linear_xent(x, 64, w, 64, 300, 64, 1000, 1, t, 64, -100, WS + big, WS + big + 4096, WS + 2 * big, need[0], None, None)
    def backward(x=P, w=Q, t=WS, lse=WS + big, g=WS + big + 4096):
        return L.guard_linear_xent_grad(x, 64, w, 64, 300, 64, 1000, 1, t, 64, -100, lse, g, 1, WS + 2 * big, WS + 3 * big, WS + 4 * big, need[1], None, None)
    for name in ("x", "w", "t"):
        for at in (0, 256):
            assert forward(**{name: WS + 2 * big + at}) == -1 and "workspace" in text(L), name
    for name in ("x", "w", "t", "lse", "g"):
        for at in (0, 256):
            assert backward(**{name: WS + 4 * big + at}) == -1 and "workspace" in text(L), name


def test_no_rows_of_an_impossible_product(L):
    """Without rows dw is all there is to clear: its size has to be one that a call with rows would take."""
    big = 1 << 40
    def backward(d=64, v=1000, w=Q, wst=64, dw=WS + 3 * big):
        return L.guard_linear_xent_grad(P, d, w, wst, 0, d, v, 1, WS, 64, -100, WS + big, WS + big + 4096, 1, None, dw, WS + 4 * big, 1 << 30, None, None)
    for bad in (dict(v=1 << 62), dict(v=1 << 60), dict(v=(1 << 30) + 8), dict(d=1 << 25, wst=1 << 25), dict(wst=56), dict(wst=68), dict(dw=Q + 160), dict(dw=WS + 4 * big)):
        assert backward(**bad) == -1, bad
        assert text(L)
    def forward(d=64, v=1000):
        return L.guard_linear_xent(P, d, Q, d, 0, d, v, 1, WS, 64, -100, WS + big, WS + big + 4096, WS + 2 * big, 1 << 30, None, None)
    assert forward() == 0 and forward(v=1 << 62) == -1 and forward(d=1 << 25) == -1


@pytest.mark.parametrize("rows,width,vocab", [(1, 8, 1), (300, 64, 1000), (8192, 4096, 131072), (40, 4096, 1 << 24), (1 << 20, 64, 5000), ((1 << 22) - 5, 128, 257), (1 << 26, 8, 300)])
def test_workspace_of_the_gradients_is_what_is_stated(L, rows, width, vocab):
    """G of a piece of the vocabulary (512 MB, or 512 bytes a row where that is more), a copy of x, dx in float32 where there are
    several pieces or few tiles, and some words a row."""
    up = lambda x, to: (x + to - 1) // to * to    # noqa: E731
    padded, columns = up(rows, 256), up(width, 256)
    held = max(min(512 << 20, padded * up(vocab, 256) * 2), padded * 512)
    need = L.guard_linear_xent_workspace_bytes(rows, width, vocab, 1)
    sums = max(padded * columns * 4, 148 // 2 * 256 * 256 * 4)
    assert padded * 512 <= need <= held + padded * width * 2 + sums + padded * 20 + 16 * 256
