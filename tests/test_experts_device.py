"""Which GPU a call of the routing and 8-bit objects runs on: that of its
tensors, whichever is current, and on no stream of another one.  Without a GPU:
the tensors are descriptions of tensors on a second one, and the library is a
recorder that looks at the current device when it is called."""
import contextlib

import pytest

import paper_2107_02103_amd as P

torch = pytest.importorskip("torch")

GPU = 1


class Tensor:
    """Shape, type and place of a contiguous tensor; views and new tensors of the same kind."""

    def __init__(self, shape, dtype=torch.float32, gpu=GPU):
        self.shape, self.dtype, self.gpu = tuple(shape), dtype, gpu
        self.device = torch.device("cuda", gpu)

    def dim(self):
        return len(self.shape)

    def __len__(self):
        return self.shape[0]

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self):
        s = [1]
        for d in self.shape[:0:-1]:
            s.insert(0, s[0] * d)
        return tuple(s)

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return True

    def contiguous(self):
        return self

    def data_ptr(self):
        return 4096

    def new_empty(self, shape, dtype=None):
        return Tensor((shape,) if isinstance(shape, int) else shape, dtype or self.dtype, self.gpu)

    def split_with_sizes(self, sizes):
        return tuple(Tensor((s,), self.dtype, self.gpu) for s in sizes)

    def view(self, *shape):
        return Tensor(shape, self.dtype, self.gpu)


class Stream:
    def __init__(self, gpu):
        self.device, self.device_index = torch.device("cuda", gpu), gpu


@pytest.fixture
def machine(monkeypatch):
    """Two GPUs, the first one current; the calls that reach the library with the GPU current at that time."""
    import paper_2107_02103_amd.experts as E
    state = {"current": 0, "calls": []}

    @contextlib.contextmanager
    def device(d):
        before, state["current"] = state["current"], torch.device(d).index if isinstance(d, str) else getattr(d, "index", d)
        try:
            yield
        finally:
            state["current"] = before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("workspace_bytes"):
                    return 256
                state["calls"].append((name, state["current"], args[0]))
                return 0
            return call

    monkeypatch.setattr(E, "_lib", Lib())
    monkeypatch.setattr(E, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(E, "_current_device", lambda: state["current"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: device(s.device))
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: Tensor(shape, dtype, device.index))
    return state


I32, I8 = torch.int32, torch.int8


def _route():
    return P.Route.from_plan(Tensor((3,), I32), Tensor((8,), I32), Tensor((4, 2), I32))


def _layer():
    return P.Int8Linear(Tensor((2, 5, 128), I8), Tensor((2, 5)), 100)


CALLS = {
    "dpc_route_plan": lambda s: P.Route(Tensor((4, 2), I32), 2, stream=s),
    "dpc_route_gather": lambda s: _route().gather(Tensor((4, 6)), stream=s),
    "dpc_route_combine": lambda s: _route().combine(Tensor((8, 6)), stream=s),
    "dpc_route_combine_bwd": lambda s: _route().combine_backward(Tensor((8, 6)), Tensor((4, 6)), stream=s),
    "dpc_quant_rows": lambda s: P.Int8Linear.from_weight(Tensor((2, 5, 100)), stream=s),
    "dpc_linear_i8": lambda s: _layer()(Tensor((4, 100)), route=_route(), stream=s),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_calls_run_on_the_device_of_their_tensors(machine, name):
    for current in (0, GPU):
        machine["current"] = current
        machine["calls"].clear()
        CALLS[name](None)
        assert machine["calls"] == [(name, GPU, 100 + GPU)]
        assert machine["current"] == current                  # the caller's choice is back


@pytest.mark.parametrize("name", list(CALLS))
def test_a_stream_of_another_device_is_refused(machine, name):
    for current in (0, GPU):
        machine["current"] = current
        with pytest.raises(ValueError, match="stream"):
            CALLS[name](Stream(0))
        assert not machine["calls"] and machine["current"] == current
    machine["current"] = 0
    CALLS[name](Stream(GPU))
    assert [c[:2] for c in machine["calls"]] == [(name, GPU)]
