"""Threads that use the operators at the same time, without a GPU: torch's device side is a stand-in."""
import threading
import time
import types


class Tensor:
    is_cuda, device = True, "cuda:0"

    def get_device(self):
        return 0

    def data_ptr(self):
        return id(self)


def test_two_first_calls_leave_one_status_word(monkeypatch):
    """Both threads are let past the check for the word together, and the first one is held up between handing the word's
    address to the library and keeping the word."""
    from paper_2605_17879_b200 import operators as ops
    together, held = threading.Barrier(2), []

    class Stream:
        def synchronize(self):
            try:
                together.wait(timeout=1.0)
            except threading.BrokenBarrierError:
                pass                            # (the other one waits elsewhere, as it should)

    class Native:
        def set_status(self, dev, address):
            held.append(address)
            if len(held) == 1:
                time.sleep(0.3)

        def embed(self, *args):
            return {}
    fake = types.SimpleNamespace(Tensor=Tensor, int32=None, zeros=lambda *a, **k: Tensor(),
                                 cuda=types.SimpleNamespace(is_current_stream_capturing=lambda: False, current_stream=lambda dev: Stream()))
    native = Native()
    monkeypatch.setattr(ops, "torch", fake)
    monkeypatch.setattr(ops, "lib", lambda: None)
    monkeypatch.setattr(ops.guard, "_native", lambda: native)
    monkeypatch.setattr(ops, "_nat", None)
    monkeypatch.setattr(ops, "_status", {})
    errors = []

    def call():
        try:
            ops.embed(Tensor(), Tensor())
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=call) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=30)
    assert not errors
    assert ops._status[0].data_ptr() == held[-1]
    assert len(held) == 1
