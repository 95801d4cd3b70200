"""Vectors of ids and the gradient of their table on the GPU against the plain ones
in 64 bits.

A lookup is one product, rounded to float32 (float64) and from there to 16 bits.
The gradient adds the rows of an id in float32, at most 1,024 of them after each
other before sums are joined in float64: off by L 2^-24 of the sum of magnitudes
for runs of L rows, 1,024 at most, a rounding for the scale and one of the result."""
import numpy as np
import pytest

import oracle.gate as og

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f64": 0.0, "f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}


def _rows(rng, n, W, t, pad=0, shift=0):
    """n rows apart by W + pad from an address that only the element divides, and as float64."""
    buf = torch.full((shift + n * (W + pad) + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + n * (W + pad)].view(n, W + pad)[:, :W]
    x.copy_(torch.from_numpy(rng.standard_normal((n, W))))
    return x, x.cpu().double().numpy()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,V,W,pad,shift", [
    (1, 1, 1, 0, 0), (7, 3, 2, 1, 1), (100, 2, 3, 0, 1), (33, 5, 7, 0, 0), (50, 9, 8, 0, 0), (64, 3, 17, 2, 1),
    (1000, 3, 240, 0, 0), (129, 1000, 241, 3, 1), (70, 70, 513, 0, 0), (10, 50000, 1600, 0, 0), (3, 4, 4099, 1, 1)])
def test_lookup(t, n, V, W, pad, shift):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n + W)
    table, plain = _rows(rng, V, W, t, pad, shift)
    ids = rng.integers(-1, V + 1, n).astype(np.int32)
    ids[:2] = (V - 1, 0)[:n]
    out = torch.full((n, W + 2), 44.0, dtype=TYPES[t], device="cuda")
    for scale in (1.0, 0.3, -64.0):
        got = P.Embedding(table, scale)(torch.from_numpy(ids).cuda(), out=out[:, :W])
        assert (out[:, W:] == 44.0).all()
        # the scale is rounded to the type of the product, then the product
        unit = STEP["f64" if t == "f64" else "f32"]
        want = og.lookup(plain, ids, scale)
        assert (np.abs(got.cpu().double().numpy() - want) <= np.abs(want) * (2.001 * unit + (STEP[t] if t != "f32" else 0)) + LEAST[t]).all()
        if scale == 1.0:
            np.testing.assert_array_equal(got.cpu().double().numpy(), want)


def _check(got, ids, dy, V, scale, t, td):
    want, mag = og.lookup_backward(ids, dy, V, scale)
    run = min(1024, np.bincount(ids[(ids >= 0) & (ids < V)], minlength=1).max())
    unit = STEP["f64" if t == "f64" else "f32"]
    bound = (run + 4) * unit * mag + 1.001 * STEP[td] * np.abs(want) + LEAST[td]
    got = got.cpu().double().numpy()
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()
    assert not got[np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V) == 0].any()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,V,W,skew", [
    (1, 1, 1, 0), (1, 70000, 5, 0), (2, 2, 3, 0), (15, 1, 8, 0), (16, 1, 7, 0), (17, 1, 9, 0), (33, 2, 240, 0),
    (64, 64, 31, 0), (100, 3, 513, 2), (1000, 1000, 16, 1), (1000, 1025, 40, 0), (5000, 3, 12, 1), (8192, 200, 33, 1),
    (8193, 200, 33, 1), (20000, 2, 240, 1), (30000, 30000, 6, 0), (3000, 1 << 20, 4, 1), (2000, (1 << 20) + 1, 2, 1),
    (4000, 300, 1601, 1), (300000, 5, 3, 1), (9000, 100000, 64, 1)])
def test_gradient(t, n, V, W, skew):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n + V)
    ids = np.minimum((V * rng.random(n) ** (1 + 3 * skew)).astype(np.int64), V - 1)
    ids[rng.random(n) < 0.05] = -1
    ids[rng.random(n) < 0.02] = V
    ids[0] = V - 1
    ids = ids.astype(np.int32)
    dy, plain = _rows(rng, n, W, t, pad=n % 3, shift=n % 2)
    dids = torch.from_numpy(ids).cuda()
    for td in dict.fromkeys((t, "f32")):
        if t == "f64" and td == "f32":
            scale = 1.0
        else:
            scale = 0.3 if n % 2 else 1.0
        buf = torch.full((V, W + 1), 33.0, dtype=TYPES[td], device="cuda")
        got = P.Embedding.gradient(dids, dy, V, scale, TYPES[td], out=buf[:, :W])
        assert (buf[:, W] == 33.0).all()
        _check(got, ids, plain, V, scale, t, td)
        again = P.Embedding.gradient(dids, dy, V, scale, TYPES[td])
        assert torch.equal(again, got)


def test_gradient_of_whole_numbers_is_exact():
    """Whole numbers whose sums fit 24 bits: every order gives the same, and a token lost or taken twice shows."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(0)
    for n, V, W in ((100000, 3, 20), (50000, 70000, 9), (16384, 16384, 130), (4096, 1, 64)):
        ids = rng.integers(0, V, n).astype(np.int32)
        dy = rng.integers(-8, 9, (n, W))
        got = P.Embedding.gradient(torch.from_numpy(ids).cuda(), torch.from_numpy(dy).float().cuda(), V)
        want, _ = og.lookup_backward(ids, dy.astype(np.float64), V)
        np.testing.assert_array_equal(got.cpu().numpy(), want)


def test_object_backward_streams_and_graphs():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(1)
    n, V, W = 20000, 300, 64
    table = torch.randn(V, W, device="cuda", dtype=torch.bfloat16)
    emb = P.Embedding(table, 8.0)
    ids = torch.from_numpy(rng.integers(0, V, n).astype(np.int32)).cuda()
    dy = torch.randn(n, W, device="cuda", dtype=torch.bfloat16)
    y, d = emb(ids), emb.backward(ids, dy)
    assert d.dtype == torch.bfloat16 and emb.backward(ids, dy, torch.float32).dtype == torch.float32
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, d2 = emb(ids, stream=s), emb.backward(ids, dy, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(d, d2)
    buf, dbuf = ids.clone(), dy.clone()
    graphs = []
    for _ in range(2):                                    # two graphs, each with a workspace of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = emb(buf), emb.backward(buf, dbuf)
        graphs.append((g, out))
    for i in range(3):
        buf.copy_(torch.from_numpy(rng.integers(-1, V, n).astype(np.int32)).cuda())
        dbuf.copy_(torch.randn(n, W, device="cuda"))
        want = emb(buf), emb.backward(buf, dbuf)
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_no_tokens():
    import paper_2107_02103_amd as P
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert P.Embedding(torch.ones(3, 5, device="cuda"))(none).shape == (0, 5)
    d = P.Embedding.gradient(none, torch.empty(0, 5, device="cuda"), 2000)
    assert d.shape == (2000, 5) and not d.any()
    ids = torch.full((70,), -1, dtype=torch.int32, device="cuda")
    assert not P.Embedding.gradient(ids, torch.full((70, 5), float("nan"), device="cuda"), 3).any()


def test_rows_past_32_bits():
    """Rows that start behind 2^31 elements, of the table and of the outputs."""
    import paper_2107_02103_amd as P
    V, W = 3, 8
    far = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    table = torch.as_strided(far, (V, W), ((1 << 30) + 512, 1))
    table.copy_(torch.arange(24.0).view(3, 8))
    ids = torch.tensor([2, 0, 1, 2], dtype=torch.int32, device="cuda")
    y = P.Embedding(table)(ids)
    assert torch.equal(y.float().cpu(), torch.arange(24.0).view(3, 8)[ids.cpu().long()])
    dy = torch.as_strided(far, (V, W), ((1 << 30) + 512, 1), 64)
    dy.copy_(torch.arange(24.0).view(3, 8) + 1)
    back = torch.as_strided(far, (V, W), ((1 << 30) + 512, 1), 128)
    P.Embedding.gradient(torch.tensor([2, 2, 0], dtype=torch.int32, device="cuda"), dy, 3, out=back)
    want = torch.zeros(3, 8)
    rows = torch.arange(24.0).view(3, 8) + 1
    want[2], want[0] = rows[0] + rows[1], rows[2]
    assert torch.equal(back.float().cpu(), want)


def test_more_than_one_dimension_of_a_launch_takes():
    """2^28 rows of 528 bytes and a gap, a wavefront to four rows: 2^32 threads and more.  (142 GB: every row is looked at.)"""
    import paper_2107_02103_amd as P
    torch.cuda.empty_cache()
    n, W = (1 << 28) + 5, 264
    if torch.cuda.mem_get_info()[0] < 190 << 30:
        pytest.skip("needs 190 GB of free memory")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[-3], ids[n // 2] = 1, -1
    table = torch.arange(1.0, 2 * W + 1, device="cuda").view(2, W).bfloat16()
    y = torch.empty(n, W, dtype=torch.bfloat16, device="cuda").fill_(-1.0)
    P.Embedding(table)(ids, out=y)
    want, odd = table[0].view(torch.int64), []
    for a in range(0, n, 1 << 23):
        rows = y[a:a + (1 << 23)].view(torch.int64)
        odd += (a + (rows != want).any(1).nonzero().flatten()).tolist()
    assert odd == [n // 2, n - 3]
    assert not y[n // 2].any() and torch.equal(y[n - 3], table[1])
    del y, ids
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,V,W", [(21, 258, 6920), (1, 64, 5003), (3, 65, 2051), (200, 130, 257), (5, 3000, 1029), (2, 70000, 260)])
def test_wide_rows_of_ids_without_tokens(n, V, W):
    """Rows of zeros that several wavefronts write, in every pair of types, with a gap behind each row."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(V)
    ids = torch.from_numpy(rng.integers(0, V, n).astype(np.int32)).cuda()
    for t, td in ((torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32),
                  (torch.float64, torch.float64), (torch.float64, torch.float32)):
        dy = torch.from_numpy(rng.integers(-4, 5, (n, W))).cuda().to(t)         # sums are exact
        out = torch.full((V, W + 1), 7.0, dtype=td, device="cuda")
        P.Embedding.gradient(ids, dy, V, dtype=td, out=out[:, :W])
        want = torch.zeros(V, W, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dy.double())
        assert torch.equal(out[:, :W].double(), want) and (out[:, W] == 7.0).all()


@pytest.mark.parametrize("t", ["f64", "f32", "bf16"])
@pytest.mark.parametrize("W", [1, 3, 9, 40, 240, 500, 1600])
def test_runs_of_every_length(t, W):
    """Ids with as many tokens as end in the middle of one part, or cross 2 to 600 of them (parts are 8 to 1,024 rows
    long): whoever joins their sums."""
    import paper_2107_02103_amd as P
    for seed, longest, n in ((0, 40, 3000), (1, 600, 20000), (2, 9000, 60000), (3, 70000, 150000)):
        if n * W > 100_000_000:
            continue
        rng = np.random.default_rng(seed + W)
        lengths = []
        while sum(lengths) < n:
            lengths.append(int(np.exp(rng.uniform(0, np.log(longest)))))
        ids = np.repeat(np.arange(len(lengths)), lengths)[:n].astype(np.int32)
        V = int(ids[-1]) + 1
        keep = rng.permutation(n)
        ids = torch.from_numpy(ids[keep]).cuda()
        dy = torch.from_numpy(rng.integers(-1, 2, (n, W)).astype(np.float32)).cuda().to(TYPES[t])   # sums are exact
        out = P.Embedding.gradient(ids, dy, V, dtype=torch.float32 if t == "bf16" else None)
        want = torch.zeros(V, W, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dy.double())
        assert torch.equal(out.double(), want), (seed, (out.double() != want).any(1).nonzero()[:4])
