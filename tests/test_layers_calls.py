"""What the Python calls of the layers do around the library's: which device is current, whose stream and arguments are passed.  No GPU: tensors on
the CPU stand in for tensors on device 1, and the library's entry points are replaced."""
import ctypes as C
import threading

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L
from paper_1704_05021_b200 import training as T


class OnDevice1(torch.Tensor):
    def get_device(self):
        return 1


def _on_device_1(t):
    return t.as_subclass(OnDevice1)


def _zeros(*shape, dtype=torch.float32):
    return _on_device_1(torch.zeros(*shape, dtype=dtype))


class Library:
    """Entry points that note which device was current and what they were given."""

    def __init__(self, state):
        self.state, self.seen, self.code = state, [], B.GD_OK

    def __getattr__(self, name):
        def call(args, stream):
            self.seen.append((name, self.state["current"], stream, bytes(args) if isinstance(args, bytes) else args))
            return self.code
        return call

    def gd_recurrence_marks_rows(self, rows, sequences, out):
        out._obj.value = rows // 64 + sequences
        return B.GD_OK


@pytest.fixture
def machine(monkeypatch):
    """Two devices, 0 current; the streams' handles are 100 + device."""
    state = {"current": 0}

    class Guard:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, state["current"] = state["current"], self.index

        def __exit__(self, *_):
            state["current"] = self.before

    lib = Library(state)
    monkeypatch.setattr(T, "_current_device", lambda: state["current"])
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(T, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(L, "load_library", lambda: lib)
    state["library"] = lib
    return state


def _session(cls, lib, **attributes):
    """A session of device 1 as its constructor leaves it, without the device."""
    s = object.__new__(cls)
    s._index, s.device, s._lib, s.workspace = 1, torch.device("cuda", 1), lib, _zeros(4096, dtype=torch.uint8)
    for name, value in attributes.items():
        setattr(s, name, value)
    return s


def _calls(lib):
    half = torch.bfloat16
    e = _session(L.EmbeddingSession, lib, vocab=10, width=8, max_tokens=4)
    n = _session(L.LayerNormSession, lib, width=8, max_rows=4, dtype=half, eps=1e-5, _code=1)
    g = _session(L.GatedLinearSession, lib, n_in=8, n_out=16, max_rows=4, dtype=half, activation="silu", w_layout="in_out", w_shape=(8, 32))
    g._bind(g.workspace)
    ids, x, stats, w = _zeros(4, dtype=torch.int64), _zeros(4, 8, dtype=half), _zeros(4), _zeros(8, 32, dtype=half)
    return [("gd_embedding_forward", lambda **k: e.forward(_zeros(10, 8), ids, out=_zeros(4, 8), **k)),
            ("gd_embedding_backward", lambda **k: e.backward(_zeros(4, 8), ids, _zeros(10, 8), **k)),
            ("gd_layer_norm_forward", lambda **k: n.forward(x, _zeros(8), _zeros(8), out=x, mean=stats, rstd=stats, **k)),
            ("gd_layer_norm_backward", lambda **k: n.backward(x, x, None, stats, stats, dx=x, dweight=_zeros(8), **k)),
            ("gd_recurrence_forward", lambda **k: L.recurrence_forward(x, x, out=x, sequences=2, marks=_zeros(2, 8), **k)),
            ("gd_recurrence_backward", lambda **k: L.recurrence_backward(x, x, x, _zeros(2, 8), x, x, sequences=2, **k)),
            ("gd_gated_forward", lambda **k: g.forward(x, w, out=_zeros(4, 16, dtype=half), **k)),
            ("gd_gated_backward", lambda **k: g.backward(_zeros(4, 16, dtype=half), x, w, _zeros(4, 32, dtype=half), dx=x, dw=w, **k))]


def test_calls_make_the_tensors_device_current_and_take_its_stream(machine):
    lib = machine["library"]
    for name, call in _calls(lib):
        call()
        assert lib.seen[-1][:3] == (name, 1, 101) and machine["current"] == 0
        call(stream=77)
        assert lib.seen[-1][:3] == (name, 1, 77) and machine["current"] == 0
    machine["current"] = 1
    for name, call in _calls(lib):
        call()
        assert lib.seen[-1][:3] == (name, 1, 101)


def test_errors_of_the_library_are_raised(machine):
    lib = machine["library"]
    lib.code = B.GD_ERR_WORKSPACE
    for name, call in _calls(lib):
        with pytest.raises(B.GdError) as e:
            call()
        assert name in str(e.value)


def test_threads_do_not_share_arguments(machine):
    """Two threads on one session: every call passes bytes of its own."""
    lib = machine["library"]
    n = _session(L.LayerNormSession, lib, width=8, max_rows=64, dtype=torch.float32, eps=1e-5, _code=0)
    rows = {r: _zeros(r, 8) for r in range(1, 65)}

    def work(which):
        for r in which:
            n.forward(rows[r], None, None, out=rows[r])

    threads = [threading.Thread(target=work, args=(range(first, 65, 2),)) for first in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    seen = [C.cast(args, C.POINTER(L._LayerNormForwardArgs)).contents for _, _, _, args in lib.seen]
    assert sorted(a.rows for a in seen) == list(range(1, 65))
    assert all(a.x == rows[a.rows].data_ptr() and a.y == a.x for a in seen)
