"""What the Python calls of the training operators do around the library's: which device is current, whose arguments are passed, what is
refused.  No GPU: tensors on the CPU stand in for tensors on device 1, and the library's entry points are replaced."""

import ctypes as C
import threading

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import training as T


class OnDevice1(torch.Tensor):
    def get_device(self):
        return 1


def _on_device_1(t):
    return t.as_subclass(OnDevice1)


class Library:
    """Entry points that note which device was current and what they were given."""

    def __init__(self, state):
        self.state, self.seen = state, []

    def __getattr__(self, name):
        def call(args, stream):
            self.seen.append((name, self.state["current"], stream))
            return B.GD_OK
        return call


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
    monkeypatch.setattr(T, "load_library", lambda: lib)
    state["library"] = lib
    return state


def _session(lib, n_in=16, n_out=24, rows=4):
    """A LinearSession of device 1 as its constructor leaves it, without the device."""
    s = object.__new__(T.LinearSession)
    s._index, s.device = 1, torch.device("cuda", 1)
    s.n_in, s.n_out, s.max_rows, s.dtype, s.activation, s.w_layout = n_in, n_out, rows, torch.bfloat16, "none", "in_out"
    s.w_shape, s._lib = (n_in, n_out), lib
    s._bind(_on_device_1(torch.zeros(4096, dtype=torch.uint8)))
    return s


def _bf16(*shape):
    return _on_device_1(torch.zeros(*shape, dtype=torch.bfloat16))


def test_calls_make_the_tensors_device_current(machine):
    lib = machine["library"]
    s = _session(lib)
    x, w, y = _bf16(4, 16), _bf16(16, 24), _bf16(4, 24)
    s.forward(x, w, out=y)
    s.backward(y, x, w, dx=_bf16(4, 16))
    s.status()
    T.cross_entropy(_on_device_1(torch.zeros(4, 8)), _on_device_1(torch.zeros(4, dtype=torch.int64)), loss=_on_device_1(torch.zeros(4)))
    a = object.__new__(T.AdamWSession)
    a._index, a._args = 1, T._AdamwArgs()
    a.step(step=1, lr=1e-3)
    assert lib.seen == [(name, 1, 101) for name in ("gd_linear_forward", "gd_linear_backward", "gd_linear_status", "gd_cross_entropy", "gd_adamw_step")]
    assert machine["current"] == 0
    machine["current"] = 1
    s.status()
    assert lib.seen[-1] == ("gd_linear_status", 1, 101)


@pytest.mark.parametrize("direction", ["forward", "backward"])
def test_threads_on_one_session_do_not_exchange_arguments(machine, direction):
    """A call into the library lets other threads run before it has read its arguments: they are its own."""
    entered, released, read = threading.Event(), threading.Event(), []

    class Slow:
        def __getattr__(self, name):
            def call(args, stream):
                if threading.current_thread() is not threading.main_thread():
                    entered.set()
                    assert released.wait(30)
                    read.append(args if isinstance(args, bytes) else C.string_at(args, 128))
                return B.GD_OK
            return call

    s = _session(Slow())
    w, mine, other = _bf16(16, 24), [_bf16(3, 16), _bf16(3, 24)], [_bf16(4, 16), _bf16(4, 24)]

    def use(x, y):
        if direction == "forward":
            s.forward(x, w, out=y)
        else:
            s.backward(y, x, w, dx=x)

    thread = threading.Thread(target=use, args=mine)
    thread.start()
    assert entered.wait(30)
    use(*other)
    released.set()
    thread.join()
    args = (T._LinearForwardArgs if direction == "forward" else T._LinearBackwardArgs).from_buffer_copy(read[0].ljust(256, b"\0"))
    assert args.m == 3 and (args.x if direction == "forward" else args.dx) == mine[0].data_ptr()
    assert (args.y if direction == "forward" else args.dy) == mine[1].data_ptr()


@pytest.mark.parametrize("as_handle", [False, True])
def test_a_result_made_by_the_call_belongs_to_its_stream(machine, monkeypatch, as_handle):
    """`out` left out with a stream given: the allocator must take its memory from that stream's, not from what the current stream has freed
    and its kernels may still be using."""
    class Stream:
        def __init__(self, handle, device=None):
            self.cuda_stream = handle

    current = [7]

    class Using:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream.cuda_stream)

        def __exit__(self, *_):
            current.pop()

    made, empty = [], torch.empty

    def make(*shape, dtype, device):
        made.append(current[-1])
        return _on_device_1(empty(*shape, dtype=dtype))

    monkeypatch.setattr(torch.cuda, "stream", Using)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(T.torch, "empty", make)
    s = _session(machine["library"])
    x, w = _bf16(4, 16), _bf16(16, 24)
    s.forward(x, w)
    s.forward(x, w, stream=55 if as_handle else Stream(55))
    assert made == [7, 55] and [seen[2] for seen in machine["library"].seen] == [101, 55]


def test_a_negative_step_is_refused(machine):
    """Not passed on as the unsigned number that its bits are."""
    a = object.__new__(T.AdamWSession)
    a._index, a._args = 1, T._AdamwArgs()
    with pytest.raises(ValueError):
        a.step(step=-1, lr=1e-3)
    assert machine["library"].seen == []


def test_refused_gradients_leave_the_old_ones():
    """A list of which one tensor is refused changes nothing: neither the type, by which all are read, nor the addresses before that one."""
    s = object.__new__(T.AdamWSession)
    s._device, s.params, s._args = torch.device("cpu"), [torch.zeros(8), torch.zeros(5)], T._AdamwArgs()
    s._tensors = (T._AdamwTensor * 2)()
    for t, p in zip(s._tensors, s.params):
        t.n = p.numel()
    first = [torch.zeros(8, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.bfloat16)]
    s.set_grads(first)
    for bad in ([torch.zeros(8), torch.zeros(4)], [torch.zeros(8), torch.zeros(5, dtype=torch.bfloat16)], [torch.zeros(8)], [torch.zeros(8).double()] * 2):
        with pytest.raises(ValueError):
            s.set_grads(bad)
        assert s._args.grad_dtype == T.GD_DTYPE_BF16 and [t.grad for t in s._tensors] == [g.data_ptr() for g in first]
        assert all(a is b for a, b in zip(s.grads, first))
    second = [torch.zeros(8), torch.zeros(5)]
    s.set_grads(second)
    assert s._args.grad_dtype == T.GD_DTYPE_FP32 and [t.grad for t in s._tensors] == [g.data_ptr() for g in second]
