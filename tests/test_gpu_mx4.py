"""Layers in microscaled 4-bit codes on the GPU against the plain ones in 64 bits.

Codes and scales are compared bit by bit, the values they stand for exactly.  A
product is summed in float32: 128 terms at a time by the matrix cores, each such sum
and its addition to the running one within 2^-23 of the magnitudes, up to 8 running
sums joined, the bias added: (K / 128 + 12) 2^-23 of the sum of magnitudes, then one
rounding of the result."""
import numpy as np
import pytest

import oracle.experts as ox
import oracle.mx4 as om

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f64": 0.0, "f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}


def check(got, want, mag, K, t):
    got = got.double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    bound = 1.001 * STEP[t] * np.abs(want) + (K / 128 + 12) * 2.0 ** -23 * mag + LEAST[t]
    bad = ~nan & ~(np.abs(got - want) <= bound)
    assert not bad.any(), (t, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("G,n,K,pad,shift", [
    (1, 1, 1, 0, 0), (1, 5, 2, 0, 1), (1, 3, 7, 1, 0), (1, 70, 16, 0, 0), (1, 9, 31, 0, 3), (2, 33, 32, 0, 0),
    (1, 33, 33, 0, 0), (1, 33, 129, 5, 1), (3, 20, 240, 0, 0), (1, 3, 255, 0, 0), (2, 3, 256, 0, 0), (1, 3, 257, 0, 0),
    (1, 19, 513, 0, 1), (1, 300, 1600, 0, 0), (2, 100, 1600, 8, 8), (1, 11, 1025, 0, 0), (1, 5, 4097, 0, 0),
    (1, 3, 8192, 0, 0), (1, 2, 16500, 0, 1)])
def test_codes_and_values(t, G, n, K, pad, shift):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n + K)
    m = G * n
    a = rng.standard_normal((m, K)) * np.exp(3 * rng.standard_normal((m, 1)))
    if m > 8:
        a[1] = 0.0
        a[2] *= 1e-38 if t != "f16" else 0.0
        a[3, K // 2] = np.inf
        a[4, K - 1] = np.nan
        a[5, 0] = -np.inf
        a[6] = np.rint(a[6] * 10) / 8                            # many ties
        a[6, ::3] = -0.0
        if t in ("f64", "f32", "bf16"):
            a[7] = 3e38 * np.sign(a[7])
        if t == "f64":
            a[8] *= 1e60                                         # infinite once rounded to float32
    buf = torch.full((shift + m * (K + pad) + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + m * (K + pad)].view(m, K + pad)[:, :K]
    x.copy_(torch.from_numpy(a))
    ld = P.mx4_ld(K)
    q = torch.full((m * ld // 2 + 64,), 99, dtype=torch.uint8, device="cuda")
    s = torch.full((m * ld // 32 + 8,), 7, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream()
    P.dpc_quant_mx4(st, P.elem_of(x.dtype), G, n, K, x, x.stride(0) if m > 1 else K, q, s)
    torch.cuda.synchronize()
    assert (q[m * ld // 2:] == 99).all() and (s[m * ld // 32:] == 7).all()
    plain = x.cpu().double().numpy()
    for g in range(G):
        want_q, want_e = om.quantise(plain[g * n:(g + 1) * n])
        codes, scales = om.pack(want_q, want_e)
        np.testing.assert_array_equal(s[:m * ld // 32].view(G, ld // 256, n, 8)[g].cpu().numpy(), scales)
        np.testing.assert_array_equal(q[:m * ld // 2].view(G, n, ld // 2)[g].cpu().numpy(), codes)
        want = om.values(want_q, want_e)[:, :K]
        for ty in TYPES:
            y = torch.full((m, K + 3), 12.0, dtype=TYPES[ty], device="cuda")
            P.dpc_values_mx4(st, P.elem_of(y.dtype), G, n, K, q, s, y, K + 3)
            assert (y[:, K:] == 12.0).all()
            got, w = y[g * n:(g + 1) * n, :K].double().cpu(), torch.from_numpy(want).to(TYPES[ty]).double()
            assert torch.equal(got.nan_to_num(nan=-5.5, posinf=1e300, neginf=-1e300),
                               w.nan_to_num(nan=-5.5, posinf=1e300, neginf=-1e300)), ty


def test_values_of_every_code_and_scale():
    import paper_2107_02103_amd as P
    q = np.tile(np.arange(256) % 16, (32, 1))
    e = np.arange(256).reshape(32, 8)
    codes, scales = om.pack(q, e)
    got = P.Mx4Rows(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 256).values(torch.float64)
    np.testing.assert_array_equal(got.cpu().numpy(), om.values(q, e))


def layer(rng, G, N, K):
    """Weights of G experts as codes on the GPU, and the values they stand for."""
    w = rng.standard_normal((G, N, K)) * np.exp(rng.standard_normal((G, N, 1)))
    packed, values = [], []
    for g in range(G):
        q, e = om.quantise(w[g])
        packed.append(om.pack(q, e))
        values.append(om.values(q, e)[:, :K])
    codes, scales = (torch.from_numpy(np.stack(a)).cuda() for a in zip(*packed))
    return codes, scales, np.stack(values), rng.standard_normal((G, N)).astype(np.float32)


def tokens(rng, m, K, t="f32", pad=0, shift=0):
    """Rows on the GPU and the values that their codes stand for."""
    buf = torch.zeros(shift + m * (K + pad) + 8, dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + m * (K + pad)].view(m, K + pad)[:, :K]
    x.copy_(torch.from_numpy(rng.standard_normal((m, K)) * np.exp(rng.standard_normal((m, 1)))))
    if m > 8:
        x[m // 3] = 0.0
        x[m // 2, K // 2] = float("nan")
    return x, om.values(*om.quantise(x.cpu().double().numpy()))[:, :K]


SIZES = [(1, 1, 1), (1, 240, 1600), (2, 3, 127), (5, 17, 128), (15, 16, 129), (16, 33, 256), (17, 15, 64), (31, 64, 640),
         (33, 65, 1000), (63, 129, 128), (64, 240, 1600), (65, 127, 257), (100, 300, 384), (127, 255, 512),
         (128, 256, 1024), (129, 257, 1600), (255, 240, 1600), (257, 128, 240), (1000, 240, 1600), (300, 1, 1600),
         (4097, 63, 130), (2049, 513, 896), (3000, 240, 256), (700, 2000, 2048), (16, 2048, 8192), (4, 512, 20000)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_layer(m, n, k):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m * 7 + n)
    codes, scales, w, bias = layer(rng, 1, n, k)
    for tx, t, b, pad, shift in (("f32", "f32", bias, 0, 0), ("bf16", "bf16", None, 3, 1), ("f16", "f16", bias, 8, 0),
                                 ("f64", "f64", bias, 0, 1), ("bf16", "bf16", bias, 0, 0), ("f32", "f64", None, 1, 3)):
        x, plain = tokens(rng, m, k, tx, pad, shift)
        if t == "f16":
            plain, x = plain / 64, x / 64
            plain = om.values(*om.quantise(x.cpu().double().numpy()))[:, :k]
        lin = P.Mx4Linear(codes, scales, k, None if b is None else torch.from_numpy(b).cuda())
        buf = torch.full((shift + m * (n + pad) + 8,), 55.0, dtype=TYPES[t], device="cuda")
        out = buf[shift:shift + m * (n + pad)].view(m, n + pad)
        lin(x, dtype=TYPES[t], out=out[:, :n])
        torch.cuda.synchronize()
        assert (out[:, n:] == 55.0).all() and (buf[:shift] == 55.0).all() and (buf[shift + m * (n + pad):] == 55.0).all()
        want, mag = om.product(plain, w[0], None if b is None else b[0])
        if t == "f16":
            assert np.nanmax(np.abs(want)) < 6e4
        check(out[:, :n], want, mag, k, t)
        coded = P.Mx4Rows.from_rows(x)
        check(lin(coded, dtype=TYPES[t]), want, mag, k, t)


GROUPED = [(1, 1, 2, 16, 32), (8, 2, 64, 100, 300), (40, 1, 3, 240, 1600), (100, 4, 5, 64, 256), (333, 2, 4, 130, 520),
           (700, 1, 2, 17, 33), (1500, 2, 8, 256, 512), (64, 8, 1, 33, 100), (2000, 1, 3, 300, 256), (50, 2, 200, 40, 64)]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("ntok,k,G,N,K", GROUPED)
def test_layers_of_experts(t, ntok, k, G, N, K):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(ntok + G)
    codes, scales, w, bias = layer(rng, G, N, K)
    x, plain = tokens(rng, ntok, K, t)
    e = (G * rng.random((ntok, k)) ** 2).astype(np.int32)
    e[rng.random((ntok, k)) < 0.1] = -1
    if G > 2:
        e[e == 1] = 0                                            # an expert without tokens
    route = P.Route(torch.from_numpy(e).cuda(), G)
    lin = P.Mx4Linear(codes, scales, K, torch.from_numpy(bias).cuda())
    y = lin(x, route=route, dtype=TYPES[t])
    off, rows, _ = ox.plan(e, G)
    want, mag = np.zeros((ntok * k, N)), np.zeros((ntok * k, N))
    for g in range(G):
        r = slice(off[g], off[g + 1])
        want[r], mag[r] = om.product(plain[rows[r] // k], w[g], bias[g])
    check(y, want, mag, K, t)
    # the same rows sorted beforehand
    y2 = lin(route.gather(x), offsets=route.offsets, dtype=TYPES[t])
    off = off[-1]
    assert torch.equal(y2[:off].nan_to_num(nan=1.0), y[:off].nan_to_num(nan=1.0)) and not y2[off:].any()
    y3 = lin(P.Mx4Rows.from_rows(x), route=route, dtype=TYPES[t])
    check(y3, want, mag, K, t)


def test_weights_and_round_trip():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(2)
    w = torch.from_numpy(rng.standard_normal((3, 50, 300))).cuda()
    lin = P.Mx4Linear.from_weight(w, torch.ones(3, 50, device="cuda", dtype=torch.float16))
    got = lin.weight().cpu().double().numpy()
    for g in range(3):
        np.testing.assert_array_equal(got[g], om.values(*om.quantise(w[g].cpu().numpy()))[:, :300])
    again = P.Mx4Linear.from_weight(lin.weight())                # what codes stand for codes to itself
    assert torch.equal(again.codes & 0x77, lin.codes & 0x77)
    assert torch.equal(again.weight(), lin.weight())


def test_scales_at_the_ends_of_their_range():
    """Blocks of 2^-100 against blocks of 2^110, which neither side holds alone in a product of scales."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(3)
    x = rng.standard_normal((20, 512))
    w = rng.standard_normal((30, 512))
    x[:, :32] *= 2.0 ** -95
    w[:, :32] *= 2.0 ** 110
    x[:, 32:] *= 2.0 ** 100
    w[:, 32:] *= 2.0 ** -96
    lin = P.Mx4Linear.from_weight(torch.from_numpy(w).cuda())
    y = lin(torch.from_numpy(x).cuda(), dtype=torch.float32)
    vx, vw = (om.values(*om.quantise(a)) for a in (x, w))
    want, mag = om.product(vx, vw)
    check(y, want, mag, 512, "f32")


def test_streams_and_graphs():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(4)
    codes, scales, _, bias = layer(rng, 4, 130, 300)
    lin = P.Mx4Linear(codes, scales, 300, torch.from_numpy(bias).cuda())
    x = torch.randn(200, 300, device="cuda")
    e = torch.from_numpy(rng.integers(-1, 4, (200, 2)).astype(np.int32)).cuda()
    route = P.Route(e, 4)
    want = lin(x, route=route)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = lin(x, route=route, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    buf, ebuf, graphs = x.clone(), e.clone(), []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = lin(buf, route=P.Route(ebuf, 4))
        graphs.append((g, out))
    for i in range(3):
        buf.copy_(torch.randn(200, 300, device="cuda"))
        ebuf.copy_(torch.from_numpy(rng.integers(-1, 4, (200, 2)).astype(np.int32)).cuda())
        want = lin(buf, route=P.Route(ebuf, 4))
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_no_rows():
    import paper_2107_02103_amd as P
    lin = P.Mx4Linear.from_weight(torch.randn(7, 40, device="cuda"))
    assert lin(torch.empty(0, 40, device="cuda")).shape == (0, 7)
    assert P.Mx4Rows.from_rows(torch.empty(0, 40, device="cuda")).values().shape == (0, 40)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k,G", [(131109, 250, 1030, 1), (131072, 33, 1024, 1), (131105, 256, 1024, 3), (66000, 17, 2049, 2)])
def test_narrow_layers_over_many_rows(t, m, n, k, G):
    """Rows that are coded and multiplied in one kernel: the same as in two (up to the order of a sum), and sampled
    rows against the plain layer."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m + n)
    codes, scales, w, bias = layer(rng, G, n, k)
    x = torch.empty(m, k + 3, dtype=TYPES[t], device="cuda")[:, :k]
    x.normal_(generator=torch.Generator("cuda").manual_seed(n))
    x[7] = 0.0
    x[m - 2, k - 1] = float("inf")
    lin = P.Mx4Linear(codes, scales, k, torch.from_numpy(bias).cuda())
    route, rows = None, np.arange(m)
    if G > 1:
        e = rng.integers(-1, G, (m, 1)).astype(np.int32)
        route = P.Route(torch.from_numpy(e).cuda(), G)
        rows = route.rows.cpu().numpy()
    for ty in (t, "f32", "f64"):
        out = torch.full((m, n + 1), 9.0, dtype=TYPES[ty], device="cuda")
        y = lin(x, route=route, dtype=TYPES[ty], out=out[:, :n])
        two = lin(P.Mx4Rows.from_rows(x), route=route, dtype=TYPES[ty])
        assert (out[:, n] == 9.0).all()
        assert torch.equal(y.isnan(), two.isnan())
        some = np.unique(np.concatenate([rng.integers(0, m, 60), [0, 31, 32, m - 1], np.flatnonzero(rows == 7),
                                         np.flatnonzero(rows == m - 2)]))
        off = [0, m] if route is None else route.offsets.tolist()
        expert = np.searchsorted(np.array(off[1:]), some, side="right")
        at = torch.from_numpy(some).cuda()
        plain = om.values(*om.quantise(x[torch.from_numpy(np.maximum(rows[some], 0)).cuda().long()].cpu().double().numpy()))[:, :k]
        want, mag = np.zeros((len(some), n)), np.zeros((len(some), n))
        for g in range(G):
            r = np.flatnonzero(expert == g)
            want[r], mag[r] = om.product(plain[r], w[g], bias[g])
        check(y[at], want, mag, k, ty)
        d = (y.double() - two.double()).abs().nan_to_num()
        # every row: twice the bound of one sum, of magnitudes under 8 sigma of k products, and a rounding
        top = 8.0 * np.sqrt(k) * float(np.abs(w).max()) * 6
        assert float(d.max()) <= 2 * (k / 128 + 12) * 2.0 ** -23 * top * np.sqrt(k) + 2.002 * STEP[ty] * float(two.nan_to_num().abs().max())
        del out, y, two, d


@pytest.mark.parametrize("K", [7680, 7681])
def test_long_rows_of_many_experts(K):
    """The longest rows that a workgroup codes itself where most experts have one (the LDS of 16 of them is 64 KiB and more
    with the sums), and longer ones."""
    test_layers_of_experts("f32", 16, 1, 64, 40, K)
    test_layers_of_experts("bf16", 16, 1, 64, 40, K)
