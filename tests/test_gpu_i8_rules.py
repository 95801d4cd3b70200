"""The sizes at which a layer's kernels change.  Layers of up to 256 channels go
from one kernel to two: short rows past 32,768, and float64 rows of more than
1,024 elements below 24,000.  Experts with few rows each go from tiles of 16
rows to larger ones.  The result is the same on both sides: the sums are exact,
and the rest is one rounding."""
import numpy as np
import pytest

import oracle.experts as ox
from tests.test_gpu_i8 import TYPES, _check, _groups, _layer, _padded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _both_sides(t, k, n, few, many, experts):
    """Rows of a layer for `many` rows and for `few` of the same ones, against the plain product."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(k + n)
    x = torch.from_numpy(rng.standard_normal((many, k)) * np.exp(rng.standard_normal((many, 1)))).to(TYPES[t]).cuda()
    x[5] = 0
    x[many - 2, k - 1] = float("nan")
    x[many - 1, 0] = float("-inf")
    qw, sw, b = _layer(rng, experts, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    qx, sx = ox.codes(x.cpu().double().numpy())
    got = {}
    for rows in (slice(many - few, many), slice(0, many)):
        m = rows.stop - rows.start
        off = np.linspace(0, m - 9, experts + 1).astype(np.int64) if experts > 1 else np.array([0, m])
        want, mag = ox.product(qx[rows], sx[rows], qw, sw, b, _groups(off, m, experts))
        y = lin(x[rows], offsets=torch.from_numpy(off.astype(np.int32)).cuda())
        _check(y, want, mag, t)
        got[m] = y
    if experts == 1:
        assert torch.equal(torch.nan_to_num(got[many][-few:], nan=1.25), torch.nan_to_num(got[few], nan=1.25))


# type, columns, rows on both sides
ONE_KERNEL = ([(t, k, 32768, 32769) for t, k in (("bf16", 240), ("f16", 59), ("bf16", 256), ("f32", 128), ("f32", 5))] +
              [("f64", k, 23999, 24000) for k in (1025, 1601, 2048)])
# experts, channels, columns, rows on both sides
FEW_ROWS = [(3, 300, 520, (64, 65)), (16, 300, 520, (128, 129)), (40, 240, 1600, (512, 513)), (20, 130, 200, (320, 321)),
            (40, 256, 2050, (512, 513))]


@pytest.mark.parametrize("experts", [1, 3])
@pytest.mark.parametrize("t,k,few,many", ONE_KERNEL)
def test_one_kernel_or_two(t, k, few, many, experts):
    _both_sides(t, k, 40 if t != "f64" else 24, few, many, experts)


@pytest.mark.parametrize("E,n,k,sizes", FEW_ROWS)
@pytest.mark.parametrize("topk", [1, 2])
def test_few_rows_of_experts(E, n, k, sizes, topk):
    # even experts, and most rows on one of them; dropped choices and experts without any
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(E + n)
    qw, sw, b = _layer(rng, E, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    for m in sizes:
        ntok = -(-m // topk)
        for share in (0.0, 0.9):
            e = rng.integers(-1, E, (ntok, topk))
            e[rng.random((ntok, topk)) < share] = E // 2
            off, rows, _ = ox.plan(e, E)
            r = P.Route(torch.from_numpy(e.astype(np.int32)).cuda(), E)
            x = torch.from_numpy(rng.standard_normal((ntok, k)).astype(np.float32)).cuda()
            x[ntok // 2] = float("nan")
            qx, sx = ox.codes(x.cpu().numpy())
            tok = np.maximum(rows, 0) // topk
            want, mag = ox.product(qx[tok], sx[tok], qw, sw, b, _groups(off, ntok * topk, E))
            _check(lin(x, route=r), want, mag, "f32")
