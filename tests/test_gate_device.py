"""Which GPU a call of the gate, of vectors of ids and of 4-bit layers runs on, and
which sizes it refuses: as tests/test_experts_device.py, with descriptions of
tensors on a second GPU and a recorder for a library."""
import contextlib

import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B
from tests.test_experts_device import GPU, Stream, Tensor

torch = pytest.importorskip("torch")
I32, U8 = torch.int32, torch.uint8


@pytest.fixture
def machine(monkeypatch):
    """Two GPUs, the first one current; the calls that reach the library with the GPU current at that time."""
    import paper_2107_02103_amd.gate as G
    import paper_2107_02103_amd.mx4 as M
    state = {"current": 0, "calls": []}

    @contextlib.contextmanager
    def device(d):
        before, state["current"] = state["current"], getattr(d, "index", d)
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

    for module in (G, M):
        monkeypatch.setattr(module, "_lib", Lib())
        monkeypatch.setattr(module, "_raw_stream", lambda d: 100 + d)
        monkeypatch.setattr(module, "_current_device", lambda: state["current"])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: device(s.device))
    return state


class Codes(Tensor):
    """Codes and what is cut from them."""

    def __getitem__(self, i):
        return Codes(((1,) + self.shape) if i is None else self.shape[1:], self.dtype, self.gpu)

    def new_empty(self, shape, dtype=None):
        return Codes((shape,) if isinstance(shape, int) else shape, dtype or self.dtype, self.gpu)

    def view(self, *shape):
        return Codes(shape, self.dtype, self.gpu)


def _rows():
    return P.Mx4Rows(Codes((4, 128), U8), Codes((1, 4, 8), U8), 100)


def _layer():
    return P.Mx4Linear(Codes((2, 5, 128), U8), Codes((2, 1, 5, 8), U8), 100)


def _route():
    return P.Route.from_plan(Tensor((3,), I32), Tensor((8,), I32), Tensor((4, 2), I32))


CALLS = {
    "dpc_gate": lambda s: P.Gate(6, 2, bias=Tensor((6,)))(Tensor((4, 6)), stream=s),
    "dpc_gate_bwd": lambda s: P.Gate(6, 2).backward(Tensor((4, 6)), Tensor((4, 2), I32), Tensor((4, 2)), stream=s),
    "dpc_embed": lambda s: P.Embedding(Tensor((3, 5)))(Tensor((4,), I32), stream=s),
    "dpc_embed_bwd": lambda s: P.Embedding(Tensor((3, 5))).backward(Tensor((4,), I32), Tensor((4, 5)), stream=s),
    "dpc_quant_mx4": lambda s: P.Mx4Rows.from_rows(Codes((4, 100)), stream=s),
    "dpc_values_mx4": lambda s: _rows().values(stream=s),
    "dpc_linear_mx4": lambda s: _layer()(Tensor((4, 100)), route=_route(), stream=s),
    "dpc_matmul_mx4": lambda s: _layer()(_rows(), route=_route(), stream=s),
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


def test_tensors_on_two_devices_are_refused(machine):
    other = dict(gpu=0)
    for call in (lambda: P.Gate(6, 2, bias=Tensor((6,), **other))(Tensor((4, 6))),
                 lambda: P.Gate(6, 2).backward(Tensor((4, 6)), Tensor((4, 2), I32, **other), Tensor((4, 2))),
                 lambda: P.Gate(6, 2).backward(Tensor((4, 6)), Tensor((4, 2), I32), Tensor((4, 2), **other)),
                 lambda: P.Embedding(Tensor((3, 5)))(Tensor((4,), I32, **other)),
                 lambda: P.Embedding.gradient(Tensor((4,), I32), Tensor((4, 5), **other), 3),
                 lambda: P.Embedding.gradient(Tensor((4,), I32), Tensor((4, 5)), 3, out=Tensor((3, 5), **other)),
                 lambda: P.Mx4Rows(Codes((4, 128), U8), Codes((1, 4, 8), U8, **other), 100),
                 lambda: P.Mx4Linear(Codes((2, 5, 128), U8), Codes((2, 1, 5, 8), U8), 100, Tensor((2, 5), **other)),
                 lambda: _layer()(Tensor((4, 100), **other), route=_route()),
                 lambda: _layer()(Tensor((4, 100)), offsets=Tensor((3,), I32, **other)),
                 lambda: _layer()(Tensor((4, 100)), route=P.Route.from_plan(Tensor((3,), I32, **other), Tensor((8,), I32, **other),
                                                                             Tensor((4, 2), I32, **other)))):
        with pytest.raises(ValueError, match="is on"):
            call()
        assert not machine["calls"]


def test_objects_refuse_sizes_past_32_bits(machine):
    BIG = 2 ** 32
    for call in (lambda: P.Gate(BIG + 6, 2), lambda: P.Gate(6, BIG + 2), lambda: P.Gate(6, 2, groups=BIG + 1),
                 lambda: P.Gate(6, 2, keep=BIG + 1), lambda: P.Gate(6, 2, best=-BIG + 1),
                 lambda: P.Gate(6, 2)(Tensor((BIG + 4, 6))),
                 lambda: P.Gate(6, 2).backward(Tensor((BIG + 4, 6)), Tensor((BIG + 4, 2), I32), Tensor((BIG + 4, 2))),
                 lambda: P.Embedding(Tensor((BIG + 3, 5))), lambda: P.Embedding(Tensor((3, BIG + 5))),
                 lambda: P.Embedding(Tensor((3, 5)))(Tensor((BIG + 4,), I32)),
                 lambda: P.Embedding.gradient(Tensor((4,), I32), Tensor((4, 5)), BIG + 3),
                 lambda: P.Embedding.gradient(Tensor((4,), I32), Tensor((4, BIG + 5)), 3),
                 lambda: P.Mx4Rows.from_rows(Codes((BIG + 4, 100))), lambda: P.Mx4Rows.from_rows(Codes((4, BIG + 100))),
                 lambda: P.Mx4Linear.from_weight(Codes((2, BIG + 5, 100))),
                 lambda: _layer()(Tensor((BIG + 4, 100)), offsets=Tensor((3,), I32))):
        with pytest.raises(P.DpcError) as e:
            call()
        assert e.value.status == B.DPC_ENOTSUP
        assert not machine["calls"]


def test_layers_refuse_what_does_not_belong_together(machine):
    layer, route = _layer(), _route()
    for call in (lambda: layer(Tensor((5, 100)), route=route), lambda: layer(Tensor((4, 99)), route=route),
                 lambda: layer(Tensor((4, 100))), lambda: layer(Tensor((4, 100)), offsets=Tensor((4,), I32)),
                 lambda: layer(Tensor((4, 100)), route=route, offsets=Tensor((3,), I32)),
                 lambda: layer(P.Mx4Rows(Codes((5, 128), U8), Codes((1, 5, 8), U8), 100), route=route),
                 lambda: layer(P.Mx4Rows(Codes((4, 128), U8), Codes((1, 4, 8), U8), 99), route=route),
                 lambda: layer(Tensor((4, 100)), route=route, out=Tensor((8, 6))),
                 lambda: layer(Tensor((4, 100)), route=route, out=Tensor((7, 5)))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        layer(Tensor((4, 100)), offsets=Tensor((3,), torch.int64))
    with pytest.raises(TypeError):
        layer(Tensor((4, 100), I32), route=route)
    with pytest.raises(TypeError):
        P.Embedding(Tensor((3, 5), I32))
    with pytest.raises(ValueError):
        P.Embedding(Tensor((3, 5))).backward(Tensor((4,), I32), Tensor((4, 6)))
    with pytest.raises(ValueError):
        P.Embedding.gradient(Tensor((4,), I32), Tensor((5, 6)), 3)
    for expert, dw in ((Tensor((4, 3), I32), Tensor((4, 2))), (Tensor((4, 2), I32), Tensor((3, 2))),
                       (Tensor((4, 2), torch.int64), Tensor((4, 2))), (Tensor((4, 2), I32), Tensor((4, 2), torch.float64))):
        with pytest.raises(ValueError):
            P.Gate(6, 2).backward(Tensor((4, 6)), expert, dw)
    with pytest.raises(ValueError, match="shape"):
        P.Gate(6, 2)(Tensor((4, 7)))
    assert not machine["calls"]
