"""Argument checks of the routing and 8-bit calls that need no GPU: every call
here is refused (or is a no-op) on the host."""
import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B

FAKE = 4096          # never dereferenced: validation fails first
I8_LD = 128


def _refused(f, base, cases):
    for kw, code in cases:
        a = dict(base)
        a.update(kw)
        with pytest.raises(P.DpcError) as e:
            f(**a)
        assert e.value.status == code, kw


def test_plan_validates_before_launch():
    nb = P.dpc_route_workspace_bytes(100, 2, 8)
    assert nb > 0 and P.dpc_route_workspace_bytes(100000, 2, 8) > 8 * 4 * 10
    for bad in ((-1, 2, 8), (4, 0, 8), (4, 65, 8), (4, 2, 0), (4, 2, 1025), (1 << 30, 2, 8)):
        assert P.dpc_route_workspace_bytes(*bad) == 0
    base = dict(stream=0, ntok=100, topk=2, nexpert=8, expert=FAKE, workspace=FAKE, workspace_bytes=nb, offsets=FAKE,
                rows=FAKE, pos=FAKE)
    _refused(P.dpc_route_plan, base, [
        (dict(ntok=-1), B.DPC_EINVAL), (dict(topk=0), B.DPC_EINVAL), (dict(nexpert=0), B.DPC_EINVAL),
        (dict(topk=65), B.DPC_ENOTSUP), (dict(nexpert=1025), B.DPC_ENOTSUP), (dict(ntok=1 << 30), B.DPC_ENOTSUP),
        (dict(expert=0), B.DPC_EINVAL), (dict(workspace=0), B.DPC_EINVAL), (dict(workspace=FAKE + 4), B.DPC_EINVAL),
        (dict(workspace_bytes=nb - 1), B.DPC_EINVAL), (dict(offsets=0), B.DPC_EINVAL), (dict(rows=0), B.DPC_EINVAL),
        (dict(pos=FAKE + 2), B.DPC_EINVAL)])


def test_rows_validate_before_launch():
    g = dict(stream=0, elem=P.DPC_ELEM_F32, ntok=4, topk=2, width=10, x=FAKE, ldx=10, weight=None, rows=FAKE,
             pos=FAKE, y=FAKE, ldy=10)
    common = [(dict(ntok=-1), B.DPC_EINVAL), (dict(topk=0), B.DPC_EINVAL), (dict(topk=65), B.DPC_ENOTSUP),
              (dict(width=0), B.DPC_EINVAL), (dict(ntok=1 << 30), B.DPC_ENOTSUP), (dict(x=0), B.DPC_EINVAL),
              (dict(x=FAKE + 2), B.DPC_EINVAL), (dict(ldx=9), B.DPC_EINVAL), (dict(weight=FAKE + 2), B.DPC_EINVAL),
              (dict(elem=7), B.DPC_EINVAL)]
    _refused(P.dpc_route_gather, g, common + [(dict(ldy=9), B.DPC_EINVAL), (dict(y=0), B.DPC_EINVAL),
                                              (dict(rows=0), B.DPC_EINVAL), (dict(pos=0), B.DPC_EINVAL)])
    c = {k: v for k, v in g.items() if k != "rows"}
    _refused(P.dpc_route_combine, c, common + [(dict(ldy=9), B.DPC_EINVAL), (dict(y=0), B.DPC_EINVAL),
                                               (dict(pos=0), B.DPC_EINVAL)])
    b = dict(stream=0, elem=P.DPC_ELEM_F64, ntok=4, topk=2, width=10, x=FAKE, ldx=10, weight=FAKE, rows=FAKE, pos=FAKE,
             dy=FAKE, lddy=10, dx=FAKE, lddx=10, dweight=FAKE)
    _refused(P.dpc_route_combine_bwd, b, common[:5] + [
        (dict(dx=None, dweight=None), B.DPC_EINVAL), (dict(x=None), B.DPC_EINVAL), (dict(dy=0), B.DPC_EINVAL),
        (dict(lddy=9), B.DPC_EINVAL), (dict(lddx=9), B.DPC_EINVAL), (dict(dweight=FAKE + 4), B.DPC_EINVAL),
        (dict(rows=0), B.DPC_EINVAL), (dict(pos=0), B.DPC_EINVAL), (dict(elem=-1), B.DPC_EINVAL)])
    # no tokens: no-ops
    P.dpc_route_gather(**{**g, "ntok": 0, "x": 0, "y": 0, "rows": 0, "pos": 0})
    P.dpc_route_combine(**{**c, "ntok": 0, "x": 0, "y": 0, "pos": 0})
    P.dpc_route_combine_bwd(**{**b, "ntok": 0, "x": 0, "dy": 0, "rows": 0, "pos": 0})


def test_8_bit_calls_validate_before_launch():
    assert B.i8_ld(1) == I8_LD and B.i8_ld(128) == I8_LD and B.i8_ld(129) == 2 * I8_LD
    q = dict(stream=0, elem=P.DPC_ELEM_BF16, nrows=4, ncols=10, x=FAKE, ldx=10, q=FAKE, scale=FAKE)
    _refused(P.dpc_quant_rows, q, [
        (dict(nrows=-1), B.DPC_EINVAL), (dict(ncols=0), B.DPC_EINVAL), (dict(ncols=131072, ldx=131072), B.DPC_ENOTSUP),
        (dict(x=0), B.DPC_EINVAL), (dict(x=FAKE + 1), B.DPC_EINVAL), (dict(ldx=9), B.DPC_EINVAL), (dict(q=0), B.DPC_EINVAL),
        (dict(q=FAKE + 8), B.DPC_EINVAL), (dict(scale=FAKE + 2), B.DPC_EINVAL), (dict(elem=4), B.DPC_EINVAL)])
    P.dpc_quant_rows(**{**q, "nrows": 0, "x": 0, "q": 0, "scale": 0})

    shared = [(dict(ntok=-1), B.DPC_EINVAL), (dict(n=0, ldy=0), B.DPC_EINVAL), (dict(k=0), B.DPC_EINVAL),
              (dict(topk=0), B.DPC_EINVAL), (dict(ngroup=0), B.DPC_EINVAL), (dict(ngroup=1025), B.DPC_ENOTSUP),
              (dict(topk=65), B.DPC_ENOTSUP), (dict(ntok=1 << 30), B.DPC_ENOTSUP),
              (dict(ntok=(1 << 26) + 1), B.DPC_ENOTSUP), (dict(n=(1 << 24) + 1, ldy=1 << 25), B.DPC_ENOTSUP),
              (dict(rows=None), B.DPC_EINVAL), (dict(offsets=None), B.DPC_EINVAL), (dict(qw=0), B.DPC_EINVAL),
              (dict(qw=FAKE + 4), B.DPC_EINVAL), (dict(sw=0), B.DPC_EINVAL), (dict(bias=FAKE + 2), B.DPC_EINVAL),
              (dict(y=0), B.DPC_EINVAL), (dict(ldy=11), B.DPC_EINVAL), (dict(y=FAKE + 2), B.DPC_EINVAL)]
    p = dict(stream=0, elem_y=P.DPC_ELEM_F32, ntok=4, topk=2, n=12, k=10, ngroup=3, qx=FAKE, sx=FAKE, rows=FAKE,
             offsets=FAKE, qw=FAKE, sw=FAKE, bias=FAKE, y=FAKE, ldy=12)
    _refused(P.dpc_matmul_i8, p, shared + [(dict(k=131072), B.DPC_ENOTSUP), (dict(qx=0), B.DPC_EINVAL),
                                           (dict(qx=FAKE + 8), B.DPC_EINVAL), (dict(sx=0), B.DPC_EINVAL),
                                           (dict(elem_y=5), B.DPC_EINVAL)])
    P.dpc_matmul_i8(**{**p, "ntok": 0, "qx": 0, "y": 0})

    nb = P.dpc_linear_i8_workspace_bytes(4, 10)
    assert nb >= 4 * I8_LD + 16 and P.dpc_linear_i8_workspace_bytes(0, 10) > 0
    for bad in ((-1, 10), (4, 0), (4, 131072)):
        assert P.dpc_linear_i8_workspace_bytes(*bad) == 0
    l = {k: v for k, v in p.items() if k not in ("qx", "sx")}
    l.update(elem_x=P.DPC_ELEM_F16, x=FAKE, ldx=10, workspace=FAKE, workspace_bytes=nb)
    _refused(P.dpc_linear_i8, l, shared + [
        (dict(k=131072, ldx=131072), B.DPC_ENOTSUP), (dict(x=0), B.DPC_EINVAL), (dict(x=FAKE + 1), B.DPC_EINVAL),
        (dict(ldx=9), B.DPC_EINVAL), (dict(workspace=0), B.DPC_EINVAL), (dict(workspace=FAKE + 8), B.DPC_EINVAL),
        (dict(workspace_bytes=nb - 1), B.DPC_EINVAL), (dict(elem_x=9), B.DPC_EINVAL)])
    P.dpc_linear_i8(**{**l, "ntok": 0, "x": 0, "y": 0})


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    f32 = lambda *s: torch.zeros(s)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="x holds"):
        P.dpc_route_gather(0, P.DPC_ELEM_F32, 4, 2, 10, f32(39), 10, None, FAKE, FAKE, FAKE, 10)
    with pytest.raises(ValueError, match="y holds"):
        P.dpc_route_gather(0, P.DPC_ELEM_F32, 4, 2, 10, FAKE, 10, None, FAKE, FAKE, f32(79), 10)
    with pytest.raises(TypeError, match="x has dtype"):
        P.dpc_route_combine(0, P.DPC_ELEM_F16, 4, 2, 10, f32(80), 10, None, FAKE, FAKE, 10)
    with pytest.raises(ValueError, match="GPU"):
        P.dpc_route_combine(0, P.DPC_ELEM_F32, 4, 2, 10, f32(80), 10, None, FAKE, FAKE, 10)
    with pytest.raises(ValueError, match="expert holds"):
        P.dpc_route_plan(0, 4, 2, 3, i32(7), FAKE, 256, FAKE, FAKE, FAKE)
    with pytest.raises(ValueError, match="dweight holds"):
        P.dpc_route_combine_bwd(0, P.DPC_ELEM_F32, 4, 2, 10, FAKE, 10, FAKE, FAKE, FAKE, FAKE, 10, FAKE, 10, f32(7))
    with pytest.raises(ValueError, match="q holds"):
        P.dpc_quant_rows(0, P.DPC_ELEM_F32, 4, 10, FAKE, 10, torch.zeros(511, dtype=torch.int8), FAKE)
    with pytest.raises(ValueError, match="qw holds"):
        P.dpc_matmul_i8(0, P.DPC_ELEM_F32, 4, 1, 12, 10, 1, FAKE, FAKE, None, None, torch.zeros(1535, dtype=torch.int8),
                        FAKE, None, FAKE, 12)
    with pytest.raises(TypeError, match="not supported"):
        P.elem_of(torch.int32)
