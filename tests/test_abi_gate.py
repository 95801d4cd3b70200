"""Argument checks of the choice of experts, of vectors of ids and of 4-bit layers
that need no GPU: every call here is refused (or is a no-op) on the host."""
import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B

torch = pytest.importorskip("torch")

FAKE = 4096          # never dereferenced: validation fails first
INF, NAN = float("inf"), float("nan")


def _refused(f, base, cases):
    for kw, code in cases:
        a = dict(base)
        a.update(kw)
        with pytest.raises(P.DpcError) as e:
            f(**a)
        assert e.value.status == code, kw


def _spec(**kw):
    v = dict(nexpert=8, topk=2, score=0, groups=1, keep=1, best=1, renorm=0, scale=1.0)
    v.update(kw)
    return P.dpc_gate_spec(*v.values())


SPECS = [(dict(nexpert=0), B.DPC_EINVAL), (dict(topk=0), B.DPC_EINVAL), (dict(topk=9), B.DPC_EINVAL),
         (dict(score=2), B.DPC_EINVAL), (dict(score=-1), B.DPC_EINVAL), (dict(groups=0), B.DPC_EINVAL),
         (dict(groups=3), B.DPC_EINVAL), (dict(keep=2), B.DPC_EINVAL), (dict(groups=2, keep=0), B.DPC_EINVAL),
         (dict(groups=2, keep=3), B.DPC_EINVAL), (dict(groups=4, keep=1, topk=3), B.DPC_EINVAL),
         (dict(best=0), B.DPC_EINVAL), (dict(best=3), B.DPC_EINVAL), (dict(scale=INF), B.DPC_EINVAL),
         (dict(scale=NAN), B.DPC_EINVAL), (dict(nexpert=1025), B.DPC_ENOTSUP), (dict(nexpert=128, topk=65), B.DPC_ENOTSUP),
         (dict(nexpert=130, groups=65), B.DPC_ENOTSUP)]


def test_gate_validates_before_launch():
    base = dict(stream=0, elem=P.DPC_ELEM_BF16, spec=_spec(), ntok=4, logits=FAKE, ldl=8, bias=None, expert=FAKE, weight=FAKE)
    _refused(P.dpc_gate, base, [(dict(spec=_spec(**kw), ldl=2000), code) for kw, code in SPECS] + [
        (dict(ntok=-1), B.DPC_EINVAL), (dict(ntok=1 << 30), B.DPC_ENOTSUP), (dict(elem=4), B.DPC_EINVAL),
        (dict(logits=0), B.DPC_EINVAL), (dict(logits=FAKE + 1), B.DPC_EINVAL), (dict(ldl=7), B.DPC_EINVAL),
        (dict(bias=FAKE + 2), B.DPC_EINVAL), (dict(expert=0), B.DPC_EINVAL), (dict(expert=FAKE + 2), B.DPC_EINVAL),
        (dict(weight=0), B.DPC_EINVAL), (dict(weight=FAKE + 2), B.DPC_EINVAL),
        (dict(elem=P.DPC_ELEM_F64, weight=FAKE + 4), B.DPC_EINVAL)])
    P.dpc_gate(**{**base, "ntok": 0, "logits": 0, "expert": 0, "weight": 0})
    base = dict(stream=0, elem=P.DPC_ELEM_F32, spec=_spec(), ntok=4, logits=FAKE, ldl=8, expert=FAKE, dweight=FAKE,
                dlogits=FAKE, lddl=8)
    _refused(P.dpc_gate_bwd, base, [(dict(spec=_spec(**kw), ldl=2000, lddl=2000), code) for kw, code in SPECS] + [
        (dict(ntok=-1), B.DPC_EINVAL), (dict(ntok=1 << 30), B.DPC_ENOTSUP), (dict(elem=-1), B.DPC_EINVAL),
        (dict(logits=0), B.DPC_EINVAL), (dict(logits=FAKE + 2), B.DPC_EINVAL), (dict(ldl=7), B.DPC_EINVAL),
        (dict(expert=0), B.DPC_EINVAL), (dict(expert=FAKE + 1), B.DPC_EINVAL), (dict(dweight=0), B.DPC_EINVAL),
        (dict(dweight=FAKE + 2), B.DPC_EINVAL), (dict(dlogits=0), B.DPC_EINVAL), (dict(dlogits=FAKE + 2), B.DPC_EINVAL),
        (dict(lddl=7), B.DPC_EINVAL)])
    P.dpc_gate_bwd(**{**base, "ntok": 0, "logits": 0, "expert": 0, "dweight": 0, "dlogits": 0})


def test_embed_validates_before_launch():
    base = dict(stream=0, elem=P.DPC_ELEM_F32, ntok=4, nid=3, width=10, ids=FAKE, table=FAKE, ldt=10, scale=1.0, y=FAKE, ldy=10)
    sizes = [(dict(ntok=-1), B.DPC_EINVAL), (dict(nid=0), B.DPC_EINVAL), (dict(width=0), B.DPC_EINVAL),
             (dict(ntok=(1 << 30) + 1), B.DPC_ENOTSUP), (dict(nid=(1 << 30) + 1), B.DPC_ENOTSUP),
             (dict(width=(1 << 31) - 127, ldt=1 << 31, ldy=1 << 31, lddy=1 << 31, lddt=1 << 31), B.DPC_ENOTSUP),
             (dict(ntok=1 << 32), B.DPC_ENOTSUP), (dict(elem=4), B.DPC_EINVAL), (dict(scale=INF), B.DPC_EINVAL),
             (dict(scale=NAN), B.DPC_EINVAL), (dict(ids=0), B.DPC_EINVAL), (dict(ids=FAKE + 2), B.DPC_EINVAL)]
    only = lambda names: [({k: v for k, v in kw.items() if k in names}, c) for kw, c in sizes]
    _refused(P.dpc_embed, base, only(base) + [
        (dict(table=0), B.DPC_EINVAL), (dict(table=FAKE + 2), B.DPC_EINVAL), (dict(ldt=9), B.DPC_EINVAL),
        (dict(y=0), B.DPC_EINVAL), (dict(y=FAKE + 2), B.DPC_EINVAL), (dict(ldy=9), B.DPC_EINVAL)])
    P.dpc_embed(**{**base, "ntok": 0, "ids": 0, "y": 0})

    nb = P.dpc_embed_bwd_workspace_bytes(P.DPC_ELEM_F32, 4, 3, 10)
    assert nb > 0
    for bad in ((4, 4, 3, 10), (0, -1, 3, 10), (0, 4, 0, 10), (0, 4, 3, 0), (0, 1 << 32, 3, 10), (0, 4, (1 << 30) + 1, 10)):
        assert P.dpc_embed_bwd_workspace_bytes(*bad) == 0
    base = dict(stream=0, elem=P.DPC_ELEM_F16, elem_d=P.DPC_ELEM_F16, ntok=4, nid=3, width=10, ids=FAKE, dy=FAKE, lddy=10,
                scale=1.0, workspace=FAKE, workspace_bytes=nb, dtable=FAKE, lddt=10)
    _refused(P.dpc_embed_bwd, base, only(base) + [
        (dict(elem_d=P.DPC_ELEM_BF16), B.DPC_EINVAL), (dict(elem_d=P.DPC_ELEM_F64), B.DPC_EINVAL),
        (dict(dy=0), B.DPC_EINVAL), (dict(dy=FAKE + 1), B.DPC_EINVAL), (dict(lddy=9), B.DPC_EINVAL),
        (dict(workspace=0), B.DPC_EINVAL), (dict(workspace=FAKE + 8), B.DPC_EINVAL), (dict(workspace_bytes=8), B.DPC_EINVAL),
        (dict(dtable=0), B.DPC_EINVAL), (dict(elem_d=P.DPC_ELEM_F32, dtable=FAKE + 2), B.DPC_EINVAL),
        (dict(lddt=9), B.DPC_EINVAL), (dict(ntok=0, dtable=0), B.DPC_EINVAL), (dict(ntok=0, workspace=0), B.DPC_EINVAL)])


def test_4_bit_calls_validate_before_launch():
    assert B.mx4_ld(1) == 256 and B.mx4_ld(256) == 256 and B.mx4_ld(257) == 512
    base = dict(stream=0, elem=P.DPC_ELEM_BF16, ngroup=2, nrows=4, ncols=10, x=FAKE, ldx=10, q=FAKE, scale=FAKE)
    cases = [(dict(ngroup=-1), B.DPC_EINVAL), (dict(nrows=-1), B.DPC_EINVAL), (dict(ncols=0), B.DPC_EINVAL),
             (dict(ncols=(1 << 20) + 1, ldx=1 << 21, ldy=1 << 21), B.DPC_ENOTSUP), (dict(nrows=1 << 30), B.DPC_ENOTSUP),
             (dict(nrows=1 << 32), B.DPC_ENOTSUP), (dict(q=0), B.DPC_EINVAL), (dict(q=FAKE + 8), B.DPC_EINVAL),
             (dict(scale=0), B.DPC_EINVAL), (dict(scale=FAKE + 4), B.DPC_EINVAL), (dict(elem=7), B.DPC_EINVAL)]
    only = lambda names: [({k: v for k, v in kw.items() if k in names}, c) for kw, c in cases]
    _refused(P.dpc_quant_mx4, base, only(base) + [(dict(x=0), B.DPC_EINVAL), (dict(x=FAKE + 1), B.DPC_EINVAL),
                                                  (dict(ldx=9), B.DPC_EINVAL)])
    for none in ("ngroup", "nrows"):
        P.dpc_quant_mx4(**{**base, none: 0, "x": 0, "q": 0, "scale": 0})
    base = {**{k: v for k, v in base.items() if k not in ("x", "ldx")}, "y": FAKE, "ldy": 10}
    _refused(P.dpc_values_mx4, base, only(base) + [(dict(y=0), B.DPC_EINVAL), (dict(y=FAKE + 1), B.DPC_EINVAL),
                                                   (dict(ldy=9), B.DPC_EINVAL)])

    shared = [(dict(ntok=-1), B.DPC_EINVAL), (dict(n=0, ldy=0), B.DPC_EINVAL), (dict(k=0), B.DPC_EINVAL),
              (dict(topk=0), B.DPC_EINVAL), (dict(ngroup=0), B.DPC_EINVAL), (dict(ngroup=1025), B.DPC_ENOTSUP),
              (dict(topk=65), B.DPC_ENOTSUP), (dict(k=(1 << 20) + 1, ldx=1 << 21), B.DPC_ENOTSUP),
              (dict(n=(1 << 24) + 1, ldy=1 << 25), B.DPC_ENOTSUP), (dict(ntok=1 << 27), B.DPC_ENOTSUP),
              (dict(ntok=1 << 32), B.DPC_ENOTSUP), (dict(elem_y=4), B.DPC_EINVAL), (dict(qw=0), B.DPC_EINVAL),
              (dict(qw=FAKE + 8), B.DPC_EINVAL), (dict(sw=0), B.DPC_EINVAL), (dict(sw=FAKE + 4), B.DPC_EINVAL),
              (dict(bias=FAKE + 2), B.DPC_EINVAL), (dict(y=0), B.DPC_EINVAL), (dict(y=FAKE + 2), B.DPC_EINVAL),
              (dict(ldy=4), B.DPC_EINVAL), (dict(rows=None), B.DPC_EINVAL), (dict(offsets=None), B.DPC_EINVAL),
              (dict(rows=FAKE + 2), B.DPC_EINVAL), (dict(offsets=FAKE + 1), B.DPC_EINVAL)]
    m = dict(stream=0, elem_y=P.DPC_ELEM_F32, ntok=4, topk=2, n=5, k=10, ngroup=3, qx=FAKE, sx=FAKE, rows=FAKE, offsets=FAKE,
             qw=FAKE, sw=FAKE, bias=None, y=FAKE, ldy=5)
    fit = lambda names: [({k: v for k, v in kw.items() if k in names}, c) for kw, c in shared]
    _refused(P.dpc_matmul_mx4, m, fit(m) + [(dict(qx=0), B.DPC_EINVAL), (dict(qx=FAKE + 4), B.DPC_EINVAL),
                                            (dict(sx=0), B.DPC_EINVAL), (dict(sx=FAKE + 4), B.DPC_EINVAL)])
    P.dpc_matmul_mx4(**{**m, "ntok": 0, "qx": 0, "sx": 0, "qw": 0, "sw": 0, "y": 0})
    nb = P.dpc_linear_mx4_workspace_bytes(4, 10)
    assert nb >= 4 * 136 and P.dpc_linear_mx4_workspace_bytes(-1, 4) == 0 and P.dpc_linear_mx4_workspace_bytes(1 << 32, 4) == 0
    assert P.dpc_linear_mx4_workspace_bytes(4, 0) == 0 and P.dpc_linear_mx4_workspace_bytes(4, (1 << 20) + 1) == 0
    lin = {**{k: v for k, v in m.items() if k not in ("qx", "sx")}, "elem_x": P.DPC_ELEM_BF16, "x": FAKE, "ldx": 10,
           "workspace": FAKE, "workspace_bytes": nb}
    _refused(P.dpc_linear_mx4, lin, fit(lin) + [
        (dict(x=0), B.DPC_EINVAL), (dict(x=FAKE + 1), B.DPC_EINVAL), (dict(ldx=9), B.DPC_EINVAL), (dict(elem_x=9), B.DPC_EINVAL),
        (dict(workspace=0), B.DPC_EINVAL), (dict(workspace=FAKE + 4), B.DPC_EINVAL), (dict(workspace_bytes=nb - 1), B.DPC_EINVAL)])
    P.dpc_linear_mx4(**{**lin, "ntok": 0, "x": 0, "workspace": 0, "qw": 0, "sw": 0, "y": 0})


def test_objects_refuse_what_is_not_on_a_gpu_or_does_not_fit():
    z, i32, u8 = torch.zeros(4, 8), torch.int32, torch.uint8
    with pytest.raises(ValueError, match="softmax or sigmoid"):
        P.Gate(8, 2, "linear")
    for bias in (torch.zeros(7), torch.zeros(8, dtype=torch.float64), torch.zeros(16)[::2], torch.zeros(8)):
        with pytest.raises(ValueError, match="bias"):
            P.Gate(8, 2, bias=bias)
    gate = P.Gate(8, 2)
    with pytest.raises(ValueError, match="GPU"):
        gate(z)
    with pytest.raises(P.DpcError):
        P.Gate(1 << 32, 2)
    with pytest.raises(ValueError, match="GPU"):
        gate.backward(z, torch.zeros(4, 2, dtype=i32), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="GPU"):
        P.Embedding(z)
    for ids in (torch.zeros(4), torch.zeros(4, dtype=torch.int64), torch.zeros(2, 2, dtype=i32), torch.zeros(8, dtype=i32)[::2]):
        with pytest.raises(ValueError, match="ids"):
            P.Embedding.gradient(ids, z, 3)
    with pytest.raises(ValueError, match="GPU"):
        P.Embedding.gradient(torch.zeros(4, dtype=i32), z, 3)
    with pytest.raises(ValueError, match="GPU"):
        P.Mx4Rows.from_rows(z)
    with pytest.raises(ValueError, match="GPU"):
        P.Mx4Linear.from_weight(z)
    codes, scales = torch.zeros(5, 128, dtype=u8), torch.zeros(1, 5, 8, dtype=u8)
    with pytest.raises(ValueError, match="GPU"):
        P.Mx4Rows(codes, scales, 200)
    for c, k in ((codes, 257), (codes.to(torch.int8), 200), (codes[:, ::2], 200), (codes[0], 200), (codes, 0)):
        with pytest.raises(ValueError, match="codes"):
            P.Mx4Rows(c, scales, k)
        with pytest.raises(ValueError):
            P.Mx4Linear(c, scales, k)
