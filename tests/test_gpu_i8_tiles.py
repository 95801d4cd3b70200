"""Every tile of the product of 8-bit codes as a routed mixture takes it: rows
that a route spreads over experts (two choices a token, some dropped, an expert
without any, groups that end inside tiles), for results of every type.  Which
tile the sizes take is checked where the rule compiles alone
(test_i8_tiles.py)."""
import numpy as np
import pytest

import oracle.experts as ox
from tests.test_gpu_i8 import TYPES, _check, _groups, _layer, _padded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EXPERTS = 4
# tokens of two choices each, channels, columns
SIZES = {(256, 256): (1399, 4000, 900), (128, 128): (2051, 4001, 700), (128, 64): (3001, 1450, 520),
         (64, 64): (1501, 300, 1300)}


@pytest.mark.parametrize("tile", list(SIZES), ids=str)
def test_tiles_of_routed_rows(tile):
    import paper_2107_02103_amd as P
    ntok, n, k = SIZES[tile]
    topk, m, ld = 2, 2 * ntok, P.i8_ld(k)
    rng = np.random.default_rng(n)
    e = rng.choice(np.array([-1, 0, 0, 0, 1, 3]), (ntok, topk))
    e[5::19] = -1                                              # tokens without any
    off, rows, _ = ox.plan(e, EXPERTS)
    assert off[2] == off[3] and off[4] < m and all(o % 64 for o in off[1:])
    r = P.Route(torch.from_numpy(e.astype(np.int32)).cuda(), EXPERTS)
    qx = rng.integers(-127, 128, (ntok, k)).astype(np.int8)
    sx = (rng.random(ntok) * 0.02).astype(np.float32)
    sx[ntok // 2] = np.nan
    qw, sw, b = _layer(rng, EXPERTS, n, k)
    tok = np.maximum(rows, 0) // topk
    want, mag = ox.product(qx[tok], sx[tok], qw, sw, b, _groups(off, m, EXPERTS))
    args = (_padded(qx, ld), torch.from_numpy(sx).cuda(), r.rows, r.offsets, _padded(qw, ld), torch.from_numpy(sw).cuda())
    for t, bias, pad, shift in (("f64", True, 0, 0), ("f64", True, 3, 1), ("f16", True, 0, 0), ("f16", False, 1, 1),
                                ("bf16", True, 5, 3), ("f32", True, 0, 0), ("f32", False, 2, 1)):
        buf = torch.full((shift + m * (n + pad) + 8,), 55.0, dtype=TYPES[t], device="cuda")
        P.dpc_matmul_i8(torch.cuda.current_stream(), P.elem_of(TYPES[t]), ntok, topk, n, k, EXPERTS, *args,
                        torch.from_numpy(b).cuda() if bias else None, buf[shift:], n + pad)
        torch.cuda.synchronize()
        with_bias, magnitude = (want, mag) if bias else ox.product(qx[tok], sx[tok], qw, sw, None, _groups(off, m, EXPERTS))
        assert np.nanmax(np.abs(with_bias)) < 6e4              # inside float16
        _check(buf[shift:shift + m * (n + pad)].view(m, n + pad)[:, :n], with_bias, magnitude, t)
        gaps = torch.ones_like(buf, dtype=torch.bool)
        gaps[shift:shift + m * (n + pad)].view(m, n + pad)[:, :n] = False
        assert (buf[gaps] == 55.0).all()


@pytest.mark.parametrize("tile", list(SIZES), ids=str)
def test_a_routed_layer_is_its_two_calls(tile):
    import paper_2107_02103_amd as P
    ntok, n, k = SIZES[tile]
    rng = np.random.default_rng(k)
    e = torch.from_numpy(rng.choice(np.array([-1, 0, 1, 3], np.int32), (ntok, 2))).cuda()
    r = P.Route(e, EXPERTS)
    qw, sw, b = _layer(rng, EXPERTS, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    x = torch.from_numpy(rng.standard_normal((ntok, k)).astype(np.float32)).cuda()
    q, s = torch.empty((ntok, P.i8_ld(k)), dtype=torch.int8, device="cuda"), torch.empty(ntok, device="cuda")
    P.dpc_quant_rows(torch.cuda.current_stream(), P.DPC_ELEM_F32, ntok, k, x, k, q, s)
    for t in ("f64", "bf16"):
        y = lin(x, route=r, dtype=TYPES[t])
        two = torch.full_like(y, 9.0)
        P.dpc_matmul_i8(torch.cuda.current_stream(), P.elem_of(y.dtype), ntok, 2, n, k, EXPERTS, q, s, r.rows, r.offsets,
                        lin.codes, lin.scales, lin.bias, two, n)
        assert torch.equal(y, two)
