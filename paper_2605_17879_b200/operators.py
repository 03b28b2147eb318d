"""Binding of the training-step operators of libguard_b200.so: token embedding, softmax cross entropy of a vocabulary
product, their gradients, and AdamW (the C ABI's last section in include/guard_b200.h).

They are the load of a node sweep (sweep_run.py) and ordinary operators besides.  Argument marshalling only, as in
guard.py: PyTorch supplies device memory and the current stream, every step runs in the library's kernels, and nothing is
recorded for autograd: a gradient is a call of its own.

Tensors that a call writes (entries of `out`, AdamW's parameters, copies and states) count as changed in place for autograd.
Calls may come from several threads, each with outputs and workspaces of its own; the interpreter lock is free meanwhile.

Errors in data (a token outside its table) cannot be raised by the call that meets them without waiting for the GPU: they
are kept in a status word per device, which sync_status() reads and clears, or in the uint32 tensor that the caller passes
as out["status"].  The first call on a device makes that word and waits for it: make it before capturing a graph.
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Dict, Optional, Sequence

import torch

from . import guard
from .guard import GUARD_OK, GuardError

STATUS_TIMEOUT, STATUS_INDEX = 2, 8
BLOCK = 256                 # elements to a scale of AdamW's 8-bit states; tensors start on such blocks of the flat states
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class _AdamwTensor(C.Structure):
    _fields_ = [("d_param", C.c_void_p), ("d_grad", C.c_void_p), ("d_copy", C.c_void_p), ("count", C.c_int64),
                ("weight_decay", C.c_float)]


_lib = None


def lib():
    """The loaded library with the operators' prototypes (raises if it has not been built)."""
    global _lib
    if _lib is None:
        L = guard.lib()
        vp, i64, f, d, i, z = C.c_void_p, C.c_int64, C.c_float, C.c_double, C.c_int, C.c_size_t
        tp = C.POINTER(_AdamwTensor)
        for name, res, args in (
                ("guard_embed", i, [vp, i, i64, vp, i64, i64, i64, i, f, vp, vp, vp]),
                ("guard_embed_grad_workspace_bytes", z, [i64, i64, i64]),
                ("guard_embed_grad", i, [vp, i64, i, vp, i, i64, i64, i64, f, i64, i, vp, vp, z, vp, vp]),
                ("guard_linear_xent_workspace_bytes", z, [i64, i64, i64, i]),
                ("guard_linear_xent", i, [vp, i64, vp, i64, i64, i64, i64, i, vp, i, i64, vp, vp, vp, z, vp, vp]),
                ("guard_linear_xent_grad", i, [vp, i64, vp, i64, i64, i64, i64, i, vp, i, i64, vp, vp, i, vp, vp, vp, z, vp, vp]),
                ("guard_debug_set_operator_wait_limit", i, [C.c_longlong]),
                ("guard_adamw_blocks", i64, [tp, i]),
                ("guard_adamw_workspace_bytes", z, [tp, i]),
                ("guard_adamw_create", i, [C.POINTER(vp), tp, i, i, i, i, d, d, d, vp, vp, vp, vp, i64, C.c_uint32, vp, z, vp]),
                ("guard_adamw_step", i, [vp, d, vp, vp, vp]),
                ("guard_adamw_steps", i, [vp, C.POINTER(i64), vp]),
                ("guard_adamw_destroy", None, [vp])):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != GUARD_OK:
        raise GuardError(rc, lib().guard_last_error(None).decode())


def _here(device: torch.device):
    return guard._HERE_CTX if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _cuda(t: torch.Tensor, what: str, device: Optional[torch.device] = None) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % what)
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, the other tensors on %s" % (what, t.device, device))
    return t.device


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError("%s must be float32, bfloat16 or float16, got %s" % (what, t.dtype))
    return code


def _contiguous(t: torch.Tensor, what: str, dtype: torch.dtype, numel: int, device: torch.device) -> int:
    _cuda(t, what, device)
    if t.dtype != dtype or not t.is_contiguous() or t.numel() != numel:
        raise ValueError("%s must be contiguous, of %s and of %d elements" % (what, dtype, numel))
    return t.data_ptr()


_status: Dict[int, torch.Tensor] = {}
_status_lock = threading.Lock()
_nat = None


def _make_status(dev: int, device) -> None:
    """The status word of a device: made once, by whichever thread comes first."""
    global _nat
    with _status_lock:
        if dev in _status:
            return
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("make the first call on a device before capturing")
        lib()
        word = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.current_stream(dev).synchronize()      # any stream may use it from now on
        _nat = guard._native()
        _nat.set_status(dev, word.data_ptr())
        _status[dev] = word


def _call(name, first, *args):
    """A native call, its device's status word in place before: the mapping of outputs."""
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        raise ValueError("expected CUDA tensors")
    dev = first.get_device()
    if dev not in _status:
        _make_status(dev, first.device)
    r = getattr(_nat, name)(first, *args)
    if r.__class__ is int:
        _check(r)
    return r


def sync_status(device=None) -> None:
    """Waits for the current stream of `device`, raises GuardError if a call before met an error in its data, and clears
    the device's status word.  (Calls still running on other streams meanwhile may set it before or after.)"""
    index = torch.device(device if device is not None else "cuda").index
    index = torch.cuda.current_device() if index is None else index
    word = _status.get(index)
    if word is None:
        return
    with torch.cuda.device(index):
        bits = int(word.item())
        if bits:
            word.zero_()
            if bits & STATUS_TIMEOUT:
                raise GuardError(-5, "a bounded wait of an operator ran out: its results are unspecified")
            raise GuardError(-1, "a token or target lies outside its table")


def debug_set_wait_limit(cycles: int) -> None:
    """Test hook: limit in clock cycles of the waits inside the cross entropy's kernels (0: the default)."""
    _check(lib().guard_debug_set_operator_wait_limit(int(cycles)))


def embed(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0,
          out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """out["out"][...] = scale * table[tokens[...]]: rows of table [rows, width], any shape of tokens.  A token outside the
    table gives a row of NaN."""
    return _call("embed", tokens, table, scale, out)


def embed_grad(grad: torch.Tensor, tokens: torch.Tensor, rows: int, *, scale: float = 1.0, padding_idx: int = -1,
               accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
               out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """out["dtable"][v] = scale * sum of grad[i] over tokens[i] == v, [rows, width] of grad's type; with accumulate, added
    to what out["dtable"] holds (rows without tokens stay as they are).  grad: [tokens, width], or contiguous of
    [..., width].  Tokens equal to padding_idx add nothing."""
    return _call("embed_grad", grad, tokens, rows, scale, padding_idx, accumulate, workspace, out)


def linear_xent(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, *, ignore_index: int = -100,
                workspace: Optional[torch.Tensor] = None, out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Softmax cross entropy of the logits x @ w.T against targets, row by row, without keeping the logits: float32
    out["loss"] and out["lse"] (the logits' log sum of exponentials, which the gradient takes).  x [rows, width] and
    w [vocab, width]: bfloat16 or float16, width a multiple of 8.  Rows whose target is ignore_index have 0 in both."""
    return _call("linear_xent", x, w, targets, ignore_index, workspace, out)


def linear_xent_grad(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, grad_loss: torch.Tensor, *,
                     ignore_index: int = -100, workspace: Optional[torch.Tensor] = None,
                     out: Optional[Dict[str, Optional[torch.Tensor]]] = None) -> Dict[str, Optional[torch.Tensor]]:
    """Gradients of (grad_loss * loss).sum(): out["dx"] and out["dw"], of the inputs' type (a missing or None entry of `out`
    is skipped).  lse: as linear_xent gave it; grad_loss: float32, one value per row, or one for all."""
    return _call("linear_xent_grad", x, w, targets, lse, grad_loss, ignore_index, workspace, out)


class AdamW:
    """AdamW over many tensors, one launch per step.

    params: contiguous float32 CUDA tensors, updated in place; grads: the buffers that a step reads, one per parameter, all
    of one type; copies: tensors of one type that receive the new parameters rounded (or None).  The tensors are kept and
    must not be moved.  weight_decay: a number, or one per tensor.

    state: {"m", "v"} of a flat layout, each parameter starting on a block of 256 elements (numel of a state:
    256 * state_blocks(params)); float32 for state_bits 32, and for 8 torch.float8_e4m3fn with {"m_scale", "v_scale"}, a
    float32 per block.  None: zeros.  step: updates made so far.

    A step may run on any stream; it waits for the constructor's work by itself, and steps must be ordered with one another.
    Neither the constructor nor steps() may be captured; finish the constructor's work before a step is.  A captured step
    holds addresses: keep the object, and all that it was given, as long as the graph is replayed.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.0, state_bits: int = 32, copies: Optional[Sequence[torch.Tensor]] = None,
                 state: Optional[Dict[str, torch.Tensor]] = None, step: int = 0, seed: int = 0):
        self._h = C.c_void_p()
        self.params, self.grads, self.copies = list(params), list(grads), None if copies is None else list(copies)
        n = len(self.params)
        if n == 0 or len(self.grads) != n or (self.copies is not None and len(self.copies) != n):
            raise ValueError("need parameters, and as many gradients and copies")
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        if len(decay) != n:
            raise ValueError("expected %d weight decays, got %d" % (n, len(decay)))
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        dev = self.device = _cuda(self.params[0], "params")
        gtype = self.grads[0].dtype
        ctype = self.copies[0].dtype if self.copies is not None else torch.float32
        table = (_AdamwTensor * n)()
        for i, p in enumerate(self.params):
            t = table[i]
            t.count, t.weight_decay = p.numel(), decay[i]
            t.d_param = _contiguous(p, "params", torch.float32, p.numel(), dev)
            t.d_grad = _contiguous(self.grads[i], "grads", gtype, p.numel(), dev)
            t.d_copy = _contiguous(self.copies[i], "copies", ctype, p.numel(), dev) if self.copies is not None else None
        gcode = _dtype(self.grads[0], "grads")
        ccode = _dtype(self.copies[0], "copies") if self.copies is not None else 0
        blocks = self.blocks = int(lib().guard_adamw_blocks(table, n))
        kinds = {"m": (torch.float32, BLOCK), "v": (torch.float32, BLOCK)} if state_bits == 32 else {
            "m": (torch.float8_e4m3fn, BLOCK), "v": (torch.float8_e4m3fn, BLOCK), "m_scale": (torch.float32, 1), "v_scale": (torch.float32, 1)}
        with _here(dev):
            own = state is None
            if own:
                state = {k: torch.zeros(blocks * per, dtype=t, device=dev) for k, (t, per) in kinds.items()}
            at = {k: _contiguous(state[k], "state[%r]" % k, t, blocks * per, dev) for k, (t, per) in kinds.items()}
            self.state = {k: state[k] for k in kinds}
            self._written = (*self.params, *(self.copies or ()), *self.state.values())
            self._wrote = guard._native().wrote
            self._ws = torch.empty(max(256, int(lib().guard_adamw_workspace_bytes(table, n))), dtype=torch.uint8, device=dev)
            _check(lib().guard_adamw_create(C.byref(self._h), table, n, gcode, ccode, state_bits, betas[0], betas[1], eps, at["m"], at["v"],
                                            at.get("m_scale"), at.get("v_scale"), step, seed & 0xFFFFFFFF, self._ws.data_ptr(),
                                            self._ws.numel(), guard._stream()))
            # (what is allocated here is handed to others in the order of this stream alone, unless the allocator hears of more)
            self._own, self._streams = [self._ws, *(self.state.values() if own else ())], {guard._stream()}
            self._made = torch.cuda.current_stream().record_event()

    @staticmethod
    def state_blocks(params: Sequence[torch.Tensor]) -> int:
        return sum((p.numel() + BLOCK - 1) // BLOCK for p in params)

    def step(self, lr, *, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One update of all parameters.  lr: a number, or a float32 CUDA tensor of one element (which a captured step reads
        at every replay); grad_scale: such a tensor too, multiplied into the gradients."""
        with _here(self.device):
            dlr = _contiguous(lr, "lr", torch.float32, 1, self.device) if isinstance(lr, torch.Tensor) else None
            gs = _contiguous(grad_scale, "grad_scale", torch.float32, 1, self.device) if grad_scale is not None else None
            stream = guard._stream()
            if stream not in self._streams:
                current = torch.cuda.current_stream()
                for t in self._own:
                    t.record_stream(current)
                if not torch.cuda.is_current_stream_capturing():      # (a capture waits for nothing outside it)
                    current.wait_event(self._made)
                    self._streams.add(stream)
            _check(lib().guard_adamw_step(self._h, 0.0 if dlr else lr, dlr, gs, stream))
        self._wrote(self._written)            # (autograd keeps versions of them)

    def steps(self) -> int:
        """Updates made so far (synchronises)."""
        n = C.c_int64()
        with _here(self.device):
            _check(lib().guard_adamw_steps(self._h, C.byref(n), guard._stream()))
        return n.value

    def close(self) -> None:
        if getattr(self, "_h", None) and _lib is not None:
            _lib.guard_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
