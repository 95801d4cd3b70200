"""Routing on the GPU against the plain one in 64 bits: plans on both sides of
every size at which their kernels change, rows of every type at widths that end
inside a chunk, strides and addresses that only the elements' size divides,
dropped choices, tokens without any, and non-finite values where nothing reads.

Bounds: a weighted row is one product, rounded once from float32 (float64), so
it is compared bit by bit.  A sum of k products has k + 1 roundings of 2^-24
(2^-53, and as much again for the plain one) of the sum of magnitudes, a dot product over W columns W / 32 + 16 in
sequence (the lanes' sums and their tree); results of 16 bits are rounded once
more, half a unit in the last place."""
import numpy as np
import pytest

import oracle.experts as ox

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f64": 2.0 ** -52, "f32": 2.0 ** -24, "f16": 2.0 ** -24, "bf16": 2.0 ** -24}
HALF = {"f64": 0.0, "f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}          # of the result, 16-bit types
LEAST = {"f64": 0.0, "f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def _choices(rng, n, k, E, drop=0.1):
    e = rng.integers(0, E, (n, k)).astype(np.int32)
    bad = rng.random((n, k)) < drop
    e[bad] = rng.choice(np.array([-1, E, -2 ** 31, 2 ** 31 - 1, -7], np.int32), int(bad.sum()))
    e[3::11] = -1                                              # tokens without any
    return e


def _guarded_plan(e, E):
    """The plan through the C call, with guards past every buffer."""
    import paper_2107_02103_amd as P
    n, k = e.shape
    nb = P.dpc_route_workspace_bytes(n, k, E)
    g = 64
    off = torch.full((E + 1 + g,), -77, dtype=torch.int32, device="cuda")
    rows = torch.full((n * k + g,), -77, dtype=torch.int32, device="cuda")
    pos = torch.full((n * k + g,), -77, dtype=torch.int32, device="cuda")
    ws = torch.full((nb + g,), 0x5A, dtype=torch.uint8, device="cuda")
    P.dpc_route_plan(torch.cuda.current_stream(), n, k, E, torch.from_numpy(e).cuda(), ws, nb, off, rows, pos)
    torch.cuda.synchronize()
    assert (off[E + 1:] == -77).all() and (rows[n * k:] == -77).all() and (pos[n * k:] == -77).all()
    assert (ws[nb:] == 0x5A).all()
    return off[:E + 1].cpu().numpy(), rows[:n * k].cpu().numpy(), pos[:n * k].cpu().numpy().reshape(n, k)


@pytest.mark.parametrize("n,k,E", [
    (1, 1, 1), (1, 2, 8), (5, 3, 2), (63, 1, 3), (64, 1, 1), (65, 1, 64), (256, 1, 2), (257, 1, 65), (1000, 4, 1024),
    (4096, 1, 2), (8192, 2, 7), (16384, 1, 3), (16385, 1, 3), (20481, 1, 1), (9000, 8, 128), (70000, 1, 1000),
    (100000, 2, 64), (4200001, 1, 2), (300, 64, 33)])
def test_plan(n, k, E):
    rng = np.random.default_rng(n + k + E)
    e = _choices(rng, n, k, E, 0.0 if n % 2 else 0.1)
    want = ox.plan(e, E)
    for _ in range(2):
        got = _guarded_plan(e, E)
        for name, g, w in zip(("offsets", "rows", "pos"), got, want):
            np.testing.assert_array_equal(g, w, err_msg=name)


@pytest.mark.parametrize("n,k,E", [(8192, 1, 5), (8193, 1, 5), (4096, 2, 70), (4097, 2, 1024), (8191, 1, 1024)])
def test_plan_where_its_kernels_change(n, k, E):
    e = _choices(np.random.default_rng(n), n, k, E)
    for g, w in zip(_guarded_plan(e, E), ox.plan(e, E)):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("n", [1, 300, 20000])
def test_plan_of_dropped_choices_alone_and_of_one_expert(n):
    off, rows, pos = _guarded_plan(np.full((n, 2), -1, np.int32), 5)
    assert not off.any() and (rows == -1).all() and (pos == -1).all()
    off, rows, pos = _guarded_plan(np.full((n, 2), 4, np.int32), 5)
    assert (off == [0, 0, 0, 0, 0, 2 * n]).all() and (rows == np.arange(2 * n)).all()


def test_plan_of_no_tokens():
    import paper_2107_02103_amd as P
    r = P.Route(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 3)
    assert r.offsets.tolist() == [0, 0, 0, 0]
    x = torch.empty((0, 5), device="cuda")
    assert r.gather(x).shape == (0, 5) and r.combine(x).shape == (0, 5)


def _strided(a, dtype, pad, shift):
    """The rows of `a` in a larger buffer: `pad` elements between rows, the first `shift` elements in; guards are NaN."""
    n, w = a.shape
    buf = torch.full((shift + n * (w + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    v = buf[shift:shift + n * (w + pad)].view(n, w + pad)[:, :w]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return buf, v


def _check(got, want, mag, n_round, t):
    """`want` in float64 from the inputs as they are stored."""
    bound = n_round * EPS[t] * 1.01 * mag + HALF[t] * np.abs(want) * 1.01 + LEAST[t]
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= bound), (t, float(np.max(err - bound)))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,k,W,pad,shift", [
    (1, 1, 1, 0, 0), (3, 2, 1, 2, 1), (9, 3, 2, 0, 1), (50, 1, 3, 0, 0), (33, 2, 5, 1, 3), (70, 4, 7, 0, 0),
    (40, 2, 8, 0, 0), (21, 2, 9, 0, 1), (300, 1, 15, 0, 0), (64, 3, 16, 0, 0), (65, 2, 17, 3, 0), (20, 8, 33, 0, 5),
    (130, 2, 64, 0, 0), (77, 2, 127, 0, 0), (77, 2, 240, 0, 0), (77, 2, 240, 16, 8), (31, 2, 257, 0, 0),
    (1, 2, 1600, 0, 0), (60, 3, 1600, 0, 1), (10, 64, 40, 0, 0), (12, 2, 4097, 0, 0), (5, 9, 8192, 0, 0),
    (3, 2, 20001, 0, 0)])
def test_rows(t, n, k, W, pad, shift):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n * 31 + W)
    E, dt = 5, TYPES[t]
    e = _choices(rng, n, k, E, 0.15)
    off, rows, pos = ox.plan(e, E)
    r = P.Route(torch.from_numpy(e).cuda(), E)
    wt = torch.float64 if t == "f64" else torch.float32
    w = torch.from_numpy(rng.standard_normal((n, k))).to(wt)
    # nothing reads the weight of a dropped choice, or an empty row
    w[torch.from_numpy(pos < 0)] = float("nan")
    wz = torch.where(torch.from_numpy(pos < 0), torch.zeros((), dtype=wt), w)
    _, x = _strided(rng.standard_normal((n, W)), dt, pad, shift)
    z = rng.standard_normal((n * k, W))
    z[off[E]:] = np.nan
    _, z = _strided(z, dt, pad, shift)
    xc, zc, wg = x.cpu().contiguous(), torch.nan_to_num(z.cpu()), w.cuda()
    x64, z64, w64 = xc.double().numpy(), zc.double().numpy(), wz.double().numpy()
    acc = torch.float64 if t == "f64" else torch.float32
    live, tok = torch.from_numpy(rows >= 0), torch.from_numpy(np.maximum(rows, 0) // k)

    # gather: bit by bit, into a strided output whose gaps stay
    for weight in (None, wg):
        buf, out = _strided(np.zeros((n * k, W)), dt, pad, shift)
        got = r.gather(x, weight, out=out)
        want = xc[tok].to(acc)
        if weight is not None:
            want = want * wz.reshape(-1)[torch.from_numpy(np.maximum(rows, 0))][:, None]
        want = torch.where(live[:, None], want, torch.zeros((), dtype=acc)).to(dt)
        assert torch.equal(got.cpu(), want)
        gaps = torch.ones_like(buf, dtype=torch.bool)
        gaps[shift:shift + n * k * (W + pad)].view(n * k, W + pad)[:, :W] = False
        assert torch.isnan(buf[gaps]).all()

    # combine
    for weight, wq in ((None, None), (wg, w64)):
        buf, out = _strided(np.zeros((n, W)), dt, pad, shift)
        got = r.combine(z, weight, out=out)
        want, mag = ox.combine(z64, pos, wq)
        _check(got, want, mag, k + 1, t)
        gaps = torch.ones_like(buf, dtype=torch.bool)
        gaps[shift:shift + n * (W + pad)].view(n, W + pad)[:, :W] = False
        assert torch.isnan(buf[gaps]).all()

    # gradient of combine
    for weight, wq in ((None, None), (wg, w64)):
        dz, dw = r.combine_backward(z, x, weight)
        want, wantw, mag = ox.combine_backward(z64, x64, rows, pos, wq)
        assert torch.equal(dz.cpu(), r.gather(x, weight).cpu())
        if weight is None:
            assert dw is None
        else:
            bound = (W / 32 + 16) * EPS[t] * mag
            assert np.all(np.abs(dw.double().cpu().numpy() - wantw) <= bound)
            none, alone = r.combine_backward(z, x, weight, need_rows=False)
            assert none is None and torch.equal(alone, dw)


def test_large_values_and_empty_experts():
    # offsets past 2^31 bytes, a row of the last token among them
    import paper_2107_02103_amd as P
    n, W = 300000, 4096
    e = torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    e[-1] = 2
    r = P.Route(e, 4)
    assert r.offsets.tolist() == [0, n - 1, n - 1, n, n]
    x = torch.zeros((n, W), dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(W, device="cuda").to(torch.bfloat16)
    x[n // 2] = 3.0
    y = r.gather(x)
    assert torch.equal(y, x)
    b = r.combine(y)
    assert torch.equal(b, x)
    d, dw = r.combine_backward(y, x, torch.ones((n, 1), device="cuda"))
    assert torch.equal(d, x)
    want = (x[[n // 2, n - 1]].double() ** 2).sum(1)
    assert torch.allclose(dw[[n // 2, n - 1], 0].double(), want, rtol=1e-5) and int((dw != 0).sum()) == 2


@pytest.mark.parametrize("t", ["f64", "f32", "bf16"])
def test_rows_past_the_caches(t):
    # over 192 MiB of aligned rows take another way than the same rows one element further apart
    import paper_2107_02103_amd as P
    n, k, W = (201 << 20) // 4 // 4096 // TYPES[t].itemsize, 4, 4096
    rng = np.random.default_rng(8)
    e = _choices(rng, n, k, 6)
    r = P.Route(torch.from_numpy(e).cuda(), 6)
    wt = torch.float64 if t == "f64" else torch.float32
    w = torch.randn((n, k), device="cuda", dtype=wt)
    x = torch.randn((n, W), device="cuda").to(TYPES[t])
    z = torch.randn((n * k, W), device="cuda").to(TYPES[t])
    apart = torch.zeros((n * k, W + 1), device="cuda", dtype=TYPES[t])[:, :W]
    apart.copy_(z)
    assert torch.equal(r.combine(z, w), r.combine(apart, w))
    assert torch.equal(r.gather(x, w), r.gather(x, w, out=torch.zeros((n * k, W + 1), device="cuda", dtype=TYPES[t])[:, :W]))
    (a, b), (c, d) = r.combine_backward(z, x, w), r.combine_backward(apart, x, w)
    assert torch.equal(a, c) and torch.equal(b, d) and torch.equal(a, r.gather(x, w))


def test_another_stream_and_repeats():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(5)
    e = torch.from_numpy(_choices(rng, 5000, 4, 9)).cuda()
    x = torch.from_numpy(rng.standard_normal((5000, 333)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.random((5000, 4)).astype(np.float32)).cuda()
    ref = P.Route(e, 9)
    ry = ref.gather(x)
    rb = ref.combine(ry, w)
    rd = ref.combine_backward(ry, rb, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        r = P.Route(e, 9, stream=s)
        y = r.gather(x, stream=s)
        b = r.combine(y, w, stream=s)
        d = r.combine_backward(y, b, w, stream=s)
        s.synchronize()
        for a, c in ((y, ry), (b, rb), (d[0], rd[0]), (d[1], rd[1]), (r.pos, ref.pos)):
            assert torch.equal(a, c)


def test_in_a_graph():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(6)
    n, k, E, W = 20000, 2, 5, 96
    e = torch.from_numpy(_choices(rng, n, k, E)).cuda()
    x = torch.from_numpy(rng.standard_normal((n, W)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.random((n, k)).astype(np.float32)).cuda()

    def step():
        r = P.Route(e, E)
        y = r.gather(x)
        b = r.combine(y, w)
        return (r.offsets, r.rows, r.pos, y, b) + r.combine_backward(y, b, w)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        e.copy_(torch.from_numpy(_choices(np.random.default_rng(i), n, k, E)))
        x.mul_(-1.1)
        want = [t.clone() for t in step()]
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c)


def test_refusals():
    import paper_2107_02103_amd as P
    e = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    r = P.Route(e, 3)
    x = torch.zeros((4, 6), device="cuda")
    with pytest.raises(ValueError):
        P.Route(e.long(), 3)
    with pytest.raises(ValueError):
        P.Route(e.cpu(), 3)
    with pytest.raises(P.DpcError):
        P.Route(e, 0)
    with pytest.raises(P.DpcError):
        P.Route(e, P.DPC_MAX_EXPERTS + 1)
    with pytest.raises(ValueError):
        r.gather(x[:3])
    with pytest.raises(ValueError):
        r.gather(x.t())
    with pytest.raises(TypeError):
        r.gather(x.int())
    with pytest.raises(ValueError):
        r.gather(x, torch.zeros((4, 2), dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        r.combine(x)
    with pytest.raises(TypeError):
        r.combine_backward(torch.zeros((8, 6), device="cuda"), x.double())
    with pytest.raises(ValueError):
        r.gather(x[:1].expand(4, 6))                     # rows on top of each other
    with pytest.raises(ValueError):
        P.Route.from_plan(r.offsets, r.rows[:-1], r.pos)
