"""Sizes past 32 bits: the routing and 8-bit calls take C ints, and a size that
does not fit one is refused before it gets there (as the same call with fewer
rows).  Nothing is launched; the library's own limits are asked with made-up
addresses, the objects with descriptions of tensors."""
import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B
from tests.test_experts_device import Tensor

torch = pytest.importorskip("torch")

FAKE = 4096          # never dereferenced: the sizes are refused first
BIG = 2 ** 32        # adds nothing to the low 32 bits of a size
I32, I8, BF16 = torch.int32, torch.int8, torch.bfloat16


def test_workspaces_of_no_size():
    for sizes in ((BIG + 8, 1, 2), (8, BIG + 1, 2), (8, 1, BIG + 2), (2 ** 31, 1, 2), (-BIG + 8, 1, 2)):
        assert P.dpc_route_workspace_bytes(*sizes) == 0
    for sizes in ((BIG + 8, 1), (8, BIG + 1), (2 ** 31, 1)):
        assert P.dpc_linear_i8_workspace_bytes(*sizes) == 0


ROWS = dict(stream=0, elem=P.DPC_ELEM_F32, ntok=4, topk=2, width=10, x=FAKE, ldx=BIG * 2, weight=None, pos=FAKE)
LAYER = dict(stream=0, elem_y=P.DPC_ELEM_F32, ntok=4, topk=1, n=12, k=10, ngroup=3, rows=FAKE, offsets=FAKE, qw=FAKE, sw=FAKE,
             bias=FAKE, y=FAKE, ldy=BIG * 2)
FUNCTIONS = [
    (P.dpc_route_plan, dict(stream=0, ntok=4, topk=2, nexpert=3, expert=FAKE, workspace=FAKE, workspace_bytes=1 << 20,
                            offsets=FAKE, rows=FAKE, pos=FAKE), ("ntok", "topk", "nexpert")),
    (P.dpc_route_gather, dict(ROWS, rows=FAKE, y=FAKE, ldy=BIG * 2), ("ntok", "topk", "width")),
    (P.dpc_route_combine, dict(ROWS, y=FAKE, ldy=BIG * 2), ("ntok", "topk", "width")),
    (P.dpc_route_combine_bwd, dict(ROWS, rows=FAKE, dy=FAKE, lddy=BIG * 2, dx=FAKE, lddx=BIG * 2, dweight=FAKE),
     ("ntok", "topk", "width")),
    (P.dpc_quant_rows, dict(stream=0, elem=P.DPC_ELEM_BF16, nrows=4, ncols=10, x=FAKE, ldx=BIG * 2, q=FAKE, scale=FAKE),
     ("nrows", "ncols")),
    (P.dpc_matmul_i8, dict(LAYER, qx=FAKE, sx=FAKE), ("ntok", "topk", "n", "k", "ngroup")),
    (P.dpc_linear_i8, dict(LAYER, elem_x=P.DPC_ELEM_F16, x=FAKE, ldx=BIG * 2, workspace=FAKE, workspace_bytes=1 << 20),
     ("ntok", "topk", "n", "k", "ngroup")),
]


@pytest.mark.parametrize("f,args,sizes", FUNCTIONS, ids=[f[0].__name__ for f in FUNCTIONS])
def test_functions_refuse_sizes_past_32_bits(f, args, sizes):
    for name in sizes:
        for value in (BIG + args[name], 2 ** 31):
            with pytest.raises(P.DpcError) as e:
                f(**dict(args, **{name: value}))
            assert e.value.status == B.DPC_ENOTSUP, (name, value)
        with pytest.raises(P.DpcError) as e:
            f(**dict(args, **{name: args[name] - BIG}))
        assert e.value.status == B.DPC_EINVAL, name


@pytest.fixture
def recorder(monkeypatch):
    """The library's calls of the objects, none of which goes on."""
    import paper_2107_02103_amd.experts as E
    calls = []

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if not name.endswith("workspace_bytes"):
                    calls.append(name)
                return 0
            return call

    monkeypatch.setattr(E, "_lib", Lib())
    monkeypatch.setattr(E, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(E, "_current_device", lambda: 1)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: Tensor(shape, dtype, device.index))
    return calls


def _route(n=4, k=2, experts=2):
    return P.Route.from_plan(Tensor((experts + 1,), I32), Tensor((n * k,), I32), Tensor((n, k), I32))


def _layer(experts=2, outer=5, inner=100):
    return P.Int8Linear(Tensor((experts, outer, P.i8_ld(inner)), I8), Tensor((experts, outer)), inner)


OBJECTS = {
    "tokens of a plan": lambda: P.Route(Tensor((BIG + 4, 1), I32), 2),
    "choices of a plan": lambda: P.Route(Tensor((4, BIG + 2), I32), 2),
    "experts of a plan": lambda: P.Route(Tensor((4, 2), I32), BIG + 2),
    "fewer than no experts": lambda: P.Route(Tensor((4, 2), I32), 2 - BIG),
    "tokens of a gather": lambda: _route(BIG + 4, 1).gather(Tensor((BIG + 4, 6))),
    "width of a gather": lambda: _route().gather(Tensor((4, BIG + 6))),
    "tokens of a combine": lambda: _route(BIG + 4, 1).combine(Tensor((BIG + 4, 6))),
    "width of a combine": lambda: _route().combine(Tensor((8, BIG + 6))),
    "width of a gradient": lambda: _route().combine_backward(Tensor((8, BIG + 6)), Tensor((4, BIG + 6))),
    "rows to code": lambda: P.Int8Linear.from_weight(Tensor((1, BIG + 5, 100))),
    "experts' rows to code": lambda: P.Int8Linear.from_weight(Tensor((2 ** 16, 2 ** 16, 1), BF16)),
    "columns to code": lambda: P.Int8Linear.from_weight(Tensor((1, 5, BIG + 100))),
    "rows of a layer": lambda: _layer(1)(Tensor((BIG + 8, 100), BF16)),
    "channels of a layer": lambda: _layer(1, BIG + 5)(Tensor((8, 100), BF16)),
    "columns of a layer": lambda: _layer(1, 5, BIG + 100)(Tensor((8, BIG + 100), BF16)),
    "experts of a layer": lambda: _layer(BIG + 1)(Tensor((8, 100)), offsets=Tensor((BIG + 2,), I32)),
}


@pytest.mark.parametrize("what", list(OBJECTS))
def test_objects_refuse_sizes_past_32_bits(recorder, what):
    with pytest.raises(P.DpcError) as e:
        OBJECTS[what]()
    assert e.value.status == B.DPC_ENOTSUP and not recorder
