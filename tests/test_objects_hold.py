"""What an object was given may be replaced or changed afterwards: a call goes by what
is there when it is made, or refuses it.  Without a GPU: descriptions of tensors, and
a recorder for a library; one test has tensors on the GPU."""
import contextlib

import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B
from tests.test_experts_device import GPU, Tensor

torch = pytest.importorskip("torch")
I32, F16, F64 = torch.int32, torch.float16, torch.float64


class Rows(Tensor):
    """Rows with a gap behind each, or (contiguous=False) an array that is not in one piece."""

    def __init__(self, shape, dtype=torch.float32, gpu=GPU, gap=0, contiguous=True):
        super().__init__(shape, dtype, gpu)
        self.gap, self.contiguous_ = gap, contiguous

    def stride(self):
        return (self.shape[1] + self.gap, 1)

    def is_contiguous(self):
        return self.contiguous_


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library, with their arguments."""
    import paper_2107_02103_amd.experts as E
    import paper_2107_02103_amd.gate as G
    import paper_2107_02103_amd.mx4 as M
    made, current = [], [GPU]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d
        try:
            yield
        finally:
            current[0] = before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("workspace_bytes"):
                    return 256
                made.append((name,) + args)
                return 0
            return call

    for module in (E, G, M):
        monkeypatch.setattr(module, "_lib", Lib())
        monkeypatch.setattr(module, "_raw_stream", lambda d: 0)
        monkeypatch.setattr(module, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    return made


def test_an_embedding_reads_the_table_that_it_has(calls):
    """The library is told the shape, type and stride of the table in place, not those of the first."""
    emb, ids = P.Embedding(Rows((300, 64))), Tensor((4,), I32)
    for table in (Rows((3, 64)), Rows((300, 64), F16), Rows((300, 8)), Rows((300, 64), gap=8), Rows((7, 5), F64)):
        emb.table = table
        calls.clear()
        out = emb(ids)
        name, _, elem, n, nid, width, _, _, ldt = calls[0][:9]
        assert (name, n, nid, width, elem, ldt) == ("dpc_embed", 4, *table.shape, B.elem_of(table.dtype), table.stride()[0])
        assert out.shape == (4, table.shape[1]) and out.dtype == table.dtype
        assert (emb.ids, emb.width) == table.shape
        emb.backward(ids, Tensor((4, emb.width), table.dtype))
        assert calls[1][4:7] == (4, *table.shape)


def test_an_embedding_refuses_a_table_that_no_constructor_takes(calls):
    emb, ids = P.Embedding(Rows((300, 64))), Tensor((4,), I32)
    for table, error in ((Rows((300, 64), I32), TypeError), (Tensor((300,)), ValueError), (Rows((300, 64), gap=-1), ValueError),
                         (torch.zeros(300, 64), ValueError), (Rows((300, 64), gpu=0), ValueError)):
        emb.table = table
        with pytest.raises(error):
            emb(ids)                                # the ids are on GPU 1
    assert not calls


def test_an_embedding_goes_on_after_a_refused_table(calls):
    first = Rows((300, 64), gap=3)
    emb, ids = P.Embedding(first), Tensor((4,), I32)
    for table in (Rows((2 ** 32, 64), gap=9), Rows((300, 64), I32)):
        emb.table = table
        with pytest.raises((P.DpcError, TypeError)):
            emb(ids)
        emb.table = first
        emb(ids)
        assert calls.pop()[2:9:2] == (B.DPC_ELEM_F32, 300, 4096, 67) and not calls


def test_an_embedding_sees_a_table_changed_in_place(calls):
    """As .data of a parameter is exchanged when its module goes to another type."""
    table = Rows((300, 64))
    emb = P.Embedding(table)
    table.shape, table.dtype = (10, 6), F16
    emb(Tensor((4,), I32))
    assert calls[0][2] == B.DPC_ELEM_F16 and calls[0][4:6] == (10, 6) and calls[0][8] == 6


BIAS = {"float64": lambda: Tensor((6,), F64), "shorter": lambda: Tensor((5,)), "a row": lambda: Tensor((1, 6)),
        "in pieces": lambda: Rows((6,), contiguous=False), "on the CPU": lambda: torch.zeros(6)}


@pytest.mark.parametrize("what", list(BIAS))
def test_a_gate_refuses_a_bias_that_no_constructor_takes(calls, what):
    gate = P.Gate(6, 2, bias=Tensor((6,)))
    gate(Tensor((4, 6)))
    gate.bias = None
    gate(Tensor((4, 6)))
    gate.bias = Tensor((6,))                        # a balancing step's new one
    gate(Tensor((4, 6)))
    assert len(calls) == 3
    gate.bias = BIAS[what]()
    with pytest.raises(ValueError, match="bias"):
        gate(Tensor((4, 6)))
    assert len(calls) == 3


def test_a_gate_sees_a_bias_changed_in_place(calls):
    gate = P.Gate(6, 2, bias=Tensor((6,)))
    gate.bias.dtype = F16
    with pytest.raises(ValueError, match="bias"):
        gate(Tensor((4, 6)))
    assert not calls


def test_a_gate_allocates_what_the_library_is_told(calls):
    """Outputs have the sizes that the specification has when the call is made."""
    gate = P.Gate(6, 2)
    gate.spec.topk = 5
    expert, weight = gate(Tensor((4, 6)))
    assert expert.shape == weight.shape == (4, 5) and (gate.nexpert, gate.topk) == (6, 5)
    with pytest.raises(ValueError, match="expert"):
        gate.backward(Tensor((4, 6)), Tensor((4, 2), I32), Tensor((4, 2)))
    gate.spec.nexpert = 7
    for call in (lambda: gate(Tensor((4, 6))), lambda: gate.backward(Tensor((4, 6)), Tensor((4, 5), I32), Tensor((4, 5)))):
        with pytest.raises(ValueError, match="logits"):
            call()
    gate.spec = B.dpc_gate_spec(8, 3, B.DPC_SCORE_SOFTMAX, 1, 1, 1, 0, 1.0)
    calls.clear()
    assert gate(Tensor((4, 8)))[0].shape == (4, 3)
    given = calls[0][3]
    given = getattr(given, "_obj", given)           # by reference
    assert (given.nexpert, given.topk) == (8, 3)
    for name in ("nexpert", "topk"):
        with pytest.raises(AttributeError):
            setattr(gate, name, 2)


class Codes(Tensor):
    """Codes and what is cut from them."""

    def __getitem__(self, i):
        return Codes(((1,) + self.shape) if i is None else self.shape[1:], self.dtype, self.gpu)

    def new_empty(self, shape, dtype=None):
        return Codes((shape,) if isinstance(shape, int) else shape, dtype or self.dtype, self.gpu)


U8 = torch.uint8


def _rows4():
    return P.Mx4Rows(Codes((4, 128), U8), Codes((1, 4, 8), U8), 100)


def _layer4():
    return P.Mx4Linear(Codes((1, 5, 128), U8), Codes((1, 1, 5, 8), U8), 100, Tensor((1, 5)))


def _refuses_others(made, names):
    """Attributes that sizes and addresses of a call follow from cannot be exchanged one by one."""
    for name in names:
        before = getattr(made, name)
        with pytest.raises(AttributeError):
            setattr(made, name, before)
        assert getattr(made, name) is before


def test_rows_and_layers_of_4_bits_keep_their_codes(calls):
    _refuses_others(_rows4(), ("codes", "scales", "cols"))
    _refuses_others(P.Mx4Rows.from_rows(Codes((4, 100))), ("codes", "scales", "cols"))
    _refuses_others(_layer4(), ("codes", "scales", "inner", "outer", "experts"))


LAYER_BIAS = {"float64": lambda: Tensor((1, 5), F64), "longer": lambda: Tensor((1, 6)), "flat": lambda: Tensor((5,)),
              "in pieces": lambda: Rows((1, 5), contiguous=False), "on the CPU": lambda: torch.zeros(1, 5),
              "elsewhere": lambda: Tensor((1, 5), gpu=0)}


@pytest.mark.parametrize("what", list(LAYER_BIAS))
def test_a_layer_of_4_bits_refuses_a_bias_that_no_constructor_takes(calls, what):
    layer = _layer4()
    layer.bias = Tensor((1, 5))
    layer(Tensor((4, 100)))
    layer(_rows4())
    layer.bias = None
    layer(Tensor((4, 100)))
    assert len(calls) == 3
    layer.bias = LAYER_BIAS[what]()
    for x in (Tensor((4, 100)), _rows4()):
        with pytest.raises(ValueError, match="bias"):
            layer(x)
    assert len(calls) == 3


def test_a_route_keeps_its_plan(calls):
    plan = Tensor((3,), I32), Tensor((8,), I32), Tensor((4, 2), I32)
    for route in (P.Route.from_plan(*plan), P.Route(Tensor((4, 2), I32), 2)):
        _refuses_others(route, ("offsets", "rows", "pos", "ntok", "topk", "nexpert"))
        route.name = "mine"                         # what a program notes at a plan is its own matter


def test_a_layer_of_8_bits_keeps_its_codes(calls):
    layer = P.Int8Linear(Tensor((2, 5, 128), torch.int8), Tensor((2, 5)), 100, Tensor((2, 5)))
    _refuses_others(layer, ("codes", "scales", "inner", "outer", "experts"))


@pytest.mark.parametrize("what", list(LAYER_BIAS))
def test_a_layer_of_8_bits_refuses_a_bias_that_no_constructor_takes(calls, what):
    layer = P.Int8Linear(Tensor((1, 5, 128), torch.int8), Tensor((1, 5)), 100, Tensor((1, 5)))
    out = Tensor((4, 5))
    layer.bias = Tensor((1, 5))
    layer(Tensor((4, 100)), out=out)
    layer.bias = None
    layer(Tensor((4, 100)), out=out)
    assert len(calls) == 2
    layer.bias = LAYER_BIAS[what]()
    with pytest.raises(ValueError, match="bias"):
        layer(Tensor((4, 100)), out=out)
    assert len(calls) == 2


@pytest.mark.gpu
def test_exchanged_tensors_on_the_gpu():
    """A table whose module goes to 16 bits, a shorter one, and other biases: results are those of new objects."""
    g = torch.Generator("cuda").manual_seed(0)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    ids = torch.tensor([0, 5, 2, -1, 7, 4], dtype=I32, device="cuda")
    module = torch.nn.Embedding(6, 40, device="cuda")
    emb = P.Embedding(module.weight, 0.5)
    emb(ids)
    module.half()
    assert emb.table is module.weight and emb.table.dtype == F16
    assert torch.equal(emb(ids), P.Embedding(module.weight.detach().clone(), 0.5)(ids)) and emb(ids).dtype == F16
    emb.table = normal(3, 50)[:, :7]
    assert torch.equal(emb(ids), P.Embedding(emb.table.clone(), 0.5)(ids))
    assert not emb(ids)[1].any() and emb.backward(ids, normal(6, 7)).shape == (3, 7)      # id 5 is none of three
    z, gate = normal(50, 12), P.Gate(12, 3, "sigmoid", bias=torch.zeros(12, device="cuda"))
    gate(z)
    gate.bias = normal(12)
    for a, b in zip(gate(z), P.Gate(12, 3, "sigmoid", bias=gate.bias)(z)):
        assert torch.equal(a, b)
    w, x = normal(9, 70), normal(5, 70)
    for kind in (P.Mx4Linear, P.Int8Linear):
        layer = kind.from_weight(w, normal(9))
        layer(x)
        layer.bias = normal(1, 9)
        assert torch.equal(layer(x), kind.from_weight(w, layer.bias[0])(x))
        layer.bias = None
        assert torch.equal(layer(x), kind.from_weight(w)(x))
