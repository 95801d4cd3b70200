"""Layers in 8-bit codes on the GPU against the plain ones in 64 bits.

The codes and scales are defined by float32 operations and compared bit by
bit.  The product's sums are exact; what follows is float64 arithmetic (a few
2^-53 of the magnitudes) and one rounding of the result to float32, 2^-24 of it,
or to 16 bits through float32 (half a unit in the last place and 2^-24)."""
import numpy as np
import pytest

import oracle.experts as ox

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f64": 0.0, "f32": 2.0 ** -24, "f16": 2.0 ** -11 + 2.0 ** -23, "bf16": 2.0 ** -8 + 2.0 ** -23}
LEAST = {"f64": 0.0, "f32": 2.0 ** -149, "f16": 2.0 ** -25 + 2.0 ** -40, "bf16": 2.0 ** -133}


def _check(got, want, mag, t):
    got = got.double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    bound = UNIT[t] * np.abs(want) * 1.001 + 8 * 2.0 ** -53 * mag + LEAST[t]
    bad = ~nan & (np.abs(got - want) > bound)
    assert not bad.any(), (t, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def _padded(q, ld):
    out = torch.zeros(q.shape[:-1] + (ld,), dtype=torch.int8)
    out[..., :q.shape[-1]] = torch.from_numpy(q)
    return out.cuda()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,K,pad,shift", [
    (1, 1, 0, 0), (5, 2, 0, 1), (3, 7, 1, 0), (70, 16, 0, 0), (9, 31, 0, 3), (33, 127, 0, 0), (33, 128, 0, 0),
    (33, 129, 5, 1), (257, 240, 0, 0), (3, 255, 0, 0), (3, 257, 0, 0), (19, 513, 0, 1), (300, 1600, 0, 0),
    (300, 1600, 8, 8), (11, 2048, 0, 0), (11, 2049, 0, 0), (5, 4097, 0, 0), (3, 8192, 0, 0), (2, 16500, 0, 1),
    (2, 131071, 0, 0)])
def test_codes(t, n, K, pad, shift):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n + K)
    a = rng.standard_normal((n, K)) * np.exp(3 * rng.standard_normal((n, 1)))
    if n > 8:
        a[1] = 0.0
        a[2] *= 1e-38 if t != "f16" else 0.0
        a[3, K // 2] = np.inf
        a[4, K - 1] = np.nan
        a[5, 0] = -np.inf
        a[6] = np.rint(a[6] * 10) / 127 * 2.0                  # many ties
        if t in ("f64", "f32", "bf16"):
            a[7] = 3e38 * np.sign(a[7])
        if t == "f64":
            a[8] *= 1e60                                        # infinite once rounded to float32
    buf = torch.full((shift + n * (K + pad) + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + n * (K + pad)].view(n, K + pad)[:, :K]
    x.copy_(torch.from_numpy(a))
    ld = P.i8_ld(K)
    q = torch.full((n * ld + 64,), 99, dtype=torch.int8, device="cuda")
    s = torch.full((n + 8,), 7.0, device="cuda")
    P.dpc_quant_rows(torch.cuda.current_stream(), P.elem_of(x.dtype), n, K, x, x.stride(0) if n > 1 else K, q, s)
    torch.cuda.synchronize()
    assert (q[n * ld:] == 99).all() and (s[n:] == 7.0).all()
    want_q, want_s = ox.codes(x.cpu().to(torch.float64).numpy())
    got = q[:n * ld].view(n, ld).cpu().numpy()
    np.testing.assert_array_equal(s[:n].cpu().numpy(), want_s)
    np.testing.assert_array_equal(got[:, :K], want_q)
    assert not got[:, K:].any()


def _layer(rng, G, N, K, low=-127):
    qw = rng.integers(low, 128, (G, N, K)).astype(np.int8)
    return qw, (rng.random((G, N)) * 0.01).astype(np.float32), rng.standard_normal((G, N)).astype(np.float32)


@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 240, 1600), (2, 3, 127), (5, 17, 128), (15, 16, 129), (16, 33, 256), (17, 15, 64), (31, 64, 640),
    (33, 65, 1000), (63, 129, 128), (64, 240, 1600), (65, 127, 257), (100, 300, 384), (127, 255, 512), (128, 256, 1024),
    (129, 257, 1600), (255, 240, 1600), (257, 128, 240), (1000, 240, 1600), (300, 1, 1600), (4097, 63, 130),
    (2049, 513, 896), (20000, 240, 256), (700, 2000, 2048)])
def test_product(m, n, k):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m * 7 + n)
    qx = rng.integers(-127, 128, (m, k)).astype(np.int8)
    sx = (rng.random(m) * 0.1).astype(np.float32)
    sx[m // 2] = np.nan if m > 4 else sx[m // 2]
    sx[m // 3] = 0.0 if m > 4 else sx[m // 3]
    qw, sw, b = _layer(rng, 1, n, k, -128)
    dqx, dqw = _padded(qx, P.i8_ld(k)), _padded(qw, P.i8_ld(k))
    dsx, dsw, db = torch.from_numpy(sx).cuda(), torch.from_numpy(sw).cuda(), torch.from_numpy(b).cuda()
    for t, bias, pad, shift in (("f32", db, 0, 0), ("bf16", None, 3, 1), ("f16", db, 8, 0), ("f64", db, 0, 1),
                                ("bf16", db, 0, 0), ("f32", None, 1, 3)):
        buf = torch.full((shift + m * (n + pad) + 8,), 55.0, dtype=TYPES[t], device="cuda")
        P.dpc_matmul_i8(torch.cuda.current_stream(), P.elem_of(TYPES[t]), m, 1, n, k, 1, dqx, dsx, None, None, dqw, dsw,
                        bias, buf[shift:], n + pad)
        torch.cuda.synchronize()
        want, mag = ox.product(qx, sx, qw, sw, None if bias is None else b)
        if t == "f16":
            keep = np.abs(np.nan_to_num(want)) < 6e4
            assert keep.all()
        _check(buf[shift:shift + m * (n + pad)].view(m, n + pad)[:, :n], want, mag, t)
        gaps = torch.ones_like(buf, dtype=torch.bool)
        gaps[shift:shift + m * (n + pad)].view(m, n + pad)[:, :n] = False
        assert (buf[gaps] == 55.0).all()


def test_product_at_the_end_of_32_bits():
    import paper_2107_02103_amd as P
    k = P.DPC_MAX_I8_COLS
    for m in (3, 40, 300):
        qx = np.full((m, k), 127, np.int8)
        qx[1] = -128
        qw = np.full((1, 40, k), -128, np.int8)
        qw[0, 2] = 127
        one = lambda *s: torch.ones(s, device="cuda")
        y = torch.empty((m, 40), dtype=torch.float64, device="cuda")
        P.dpc_matmul_i8(torch.cuda.current_stream(), P.DPC_ELEM_F64, m, 1, 40, k, 1, _padded(qx, P.i8_ld(k)), one(m),
                        None, None, _padded(qw, P.i8_ld(k)), one(1, 40), None, y, 40)
        want, _ = ox.product(qx, np.ones(m), qw, np.ones((1, 40)))
        assert np.array_equal(y.cpu().numpy(), want) and want.max() == 128 * 128 * k


def test_large_and_small_scales():
    # the product of sum and one scale leaves float32's range, the result does not
    import paper_2107_02103_amd as P
    x = torch.tensor([[3e38, 1e38, -2e38], [1e-30, 3e-31, 5e-30]], device="cuda")
    lin = P.Int8Linear.from_weight(torch.tensor([[1e-3, 0.5e-3, 1e-3], [1e-10, 1e-9, 1e-10]], device="cuda"))
    y = lin(x)
    qx, sx = ox.codes(x.cpu().numpy())
    want, mag = ox.product(qx, sx, lin.codes[:, :, :3].cpu().numpy(), lin.scales.cpu().numpy())
    _check(y, want, mag, "f32")
    assert np.isfinite(want).all() and (np.abs(want) > 0).all()


def _groups(off, m, G):
    g = np.full(m, -1)
    for e in range(G):
        g[off[e]:off[e + 1]] = e
    return g


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("ntok,topk,G,n,k", [
    (1, 1, 1, 5, 3), (1, 2, 64, 240, 1600), (8, 2, 64, 130, 256), (16, 4, 3, 48, 130), (40, 1, 2, 240, 1600),
    (77, 3, 5, 33, 100), (300, 1, 3, 240, 320), (300, 2, 70, 65, 129), (500, 2, 1000, 20, 64), (1000, 1, 3, 256, 1024),
    (2100, 2, 4, 240, 256), (5000, 1, 3, 240, 1600), (900, 2, 9, 520, 512)])
def test_layer_of_experts(t, ntok, topk, G, n, k):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(ntok + G)
    e = np.minimum(rng.integers(-1, G, (ntok, topk)), rng.integers(0, G, (ntok, topk))).astype(np.int32)
    off, rows, pos = ox.plan(e, G)
    r = P.Route(torch.from_numpy(e).cuda(), G)
    x = torch.from_numpy(rng.standard_normal((ntok, k)) * np.exp(rng.standard_normal((ntok, 1)))).to(TYPES[t]).cuda()
    if ntok > 10:
        x[3] = 0
        x[7, k // 2] = float("nan")
    qw, sw, b = _layer(rng, G, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    qx, sx = ox.codes(x.cpu().double().numpy())
    tok = np.maximum(rows, 0) // topk
    want, mag = ox.product(qx[tok], sx[tok], qw, sw, b, _groups(off, ntok * topk, G))
    out = "f32" if t == "f16" else t
    y = lin(x, route=r, dtype=TYPES[out])
    _check(y, want, mag, out)
    # rows that are sorted already
    xs = x[torch.from_numpy(tok).cuda()]
    _check(lin(xs, offsets=r.offsets, dtype=TYPES[out]), want, mag, out)
    # in two calls, with the same result
    ld = P.i8_ld(k)
    q = torch.empty((ntok, ld), dtype=torch.int8, device="cuda")
    s = torch.empty(ntok, device="cuda")
    P.dpc_quant_rows(torch.cuda.current_stream(), P.elem_of(x.dtype), ntok, k, x, k, q, s)
    two = torch.full_like(y, 9.0)
    P.dpc_matmul_i8(torch.cuda.current_stream(), P.elem_of(y.dtype), ntok, topk, n, k, G, q, s, r.rows, r.offsets,
                    lin.codes, lin.scales, lin.bias, two, n)
    assert torch.equal(torch.nan_to_num(two, nan=1.25), torch.nan_to_num(y, nan=1.25))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n,k,pad,shift", [
    (1, 240, 1600, 0, 0), (1, 7, 3, 0, 1), (3, 240, 1600, 0, 0), (16, 512, 2048, 0, 0), (17, 100, 99, 1, 0),
    (48, 240, 240, 0, 0), (129, 240, 1600, 0, 0), (1111, 240, 1600, 4, 0), (1111, 256, 1601, 0, 3), (5000, 33, 130, 0, 0),
    (9000, 240, 2049, 0, 0), (70, 1600, 240, 0, 0), (4100, 250, 5000, 0, 0)])
def test_layer(t, m, n, k, pad, shift):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m + n + k)
    buf = torch.full((shift + m * (k + pad) + 8,), float("nan"), dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + m * (k + pad)].view(m, k + pad)[:, :k]
    x.copy_(torch.from_numpy(rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))))
    if m > 40:
        x[39] = 0
        x[m - 1, k - 1] = float("inf")
    W = torch.from_numpy(rng.standard_normal((n, k)) / np.sqrt(k)).to(TYPES[t]).cuda()
    b = torch.from_numpy(rng.standard_normal(n)).cuda()
    lin = P.Int8Linear.from_weight(W, b)
    qw, sw = ox.codes(W.cpu().double().numpy())
    np.testing.assert_array_equal(lin.codes[0, :, :k].cpu().numpy(), qw)
    qx, sx = ox.codes(x.cpu().double().numpy())
    want, mag = ox.product(qx, sx, qw[None], sw[None], b.float().cpu().double().numpy()[None])
    for out in ("f32", t):
        y = lin(x, dtype=TYPES[out])
        _check(y, want, mag, out)
        assert torch.equal(torch.nan_to_num(y, nan=1.25), torch.nan_to_num(lin(x, dtype=TYPES[out]), nan=1.25))
    # the codes stand for x and W to half a step: error of the layer against the product itself
    ok = np.isfinite(sx)
    ref = x.cpu().double().numpy()[ok] @ W.cpu().double().numpy().T + b.cpu().numpy()
    xa, wa = np.abs(x.cpu().double().numpy()[ok]), np.abs(W.cpu().double().numpy())
    half_x, half_w = 0.501 * sx[ok].astype(float)[:, None], 0.501 * sw.astype(float)[None, :]
    bound = half_x * wa.sum(1) + xa.sum(1)[:, None] * half_w + k * half_x * half_w + 1e-5
    assert (np.abs(lin(x, dtype=torch.float64).cpu().numpy()[ok] - ref) <= bound).all()


def test_gradient_is_the_product_with_the_transposed_weights():
    # y is linear in x at fixed codes of W: its gradient in x is dy W, here with the codes of W^T
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(4)
    W = torch.from_numpy(rng.standard_normal((240, 320)) / 18).cuda()
    back = P.Int8Linear.from_weight(W.t())
    dy = torch.from_numpy(rng.standard_normal((70, 240))).cuda()
    dx = back(dy)
    qd, sd = ox.codes(dy.cpu().numpy())
    qt, st = ox.codes(W.t().cpu().numpy())
    want, mag = ox.product(qd, sd, qt[None], st[None])
    _check(dx, want, mag, "f64")
    exact = dy.cpu().numpy() @ W.cpu().numpy()
    assert np.linalg.norm(want - exact) < 0.02 * np.linalg.norm(exact)


def test_in_a_graph_and_on_another_stream():
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(7)
    lins, xs, e = [], [], torch.from_numpy(rng.integers(0, 3, (700, 2)).astype(np.int32)).cuda()
    for n, k in ((240, 1600), (512, 300)):
        lins.append(P.Int8Linear.from_weight(torch.from_numpy(rng.standard_normal((3, n, k))).cuda()))
        xs.append(torch.from_numpy(rng.standard_normal((700, k)).astype(np.float32)).cuda())
    few = P.Int8Linear.from_weight(torch.from_numpy(rng.standard_normal((1000, 500))).cuda())
    xf = torch.from_numpy(rng.standard_normal((4, 500)).astype(np.float32)).cuda()

    def step():
        r = P.Route(e, 3)
        return [l(x, route=r) for l, x in zip(lins, xs)] + [few(xf)]

    side = torch.cuda.Stream()
    want = step()
    torch.cuda.synchronize()
    got = [few(xf, stream=side)]
    side.synchronize()
    assert torch.equal(got[0], want[2])
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        e.copy_(torch.from_numpy(rng.integers(-1, 3, (700, 2)).astype(np.int32)))
        for x in xs + [xf]:
            x.mul_(-1.3)
        want = [w.clone() for w in step()]
        g.replay()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c)


def test_refusals():
    import paper_2107_02103_amd as P
    W = torch.zeros((3, 8, 40), device="cuda")
    lin = P.Int8Linear.from_weight(W)
    x = torch.zeros((4, 40), device="cuda")
    r = P.Route(torch.zeros((4, 1), dtype=torch.int32, device="cuda"), 2)
    with pytest.raises(ValueError):
        lin(x)                                              # several experts, no route
    with pytest.raises(ValueError):
        lin(x, route=r)                                     # a route to two experts, layers of three
    with pytest.raises(ValueError):
        lin(x[:, :39], offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        lin(x, offsets=torch.zeros(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        lin(x.cpu(), offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        lin(x.int(), offsets=torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        P.Int8Linear(lin.codes, lin.scales, 200)            # codes of another width
    with pytest.raises(ValueError):
        P.Int8Linear(lin.codes, lin.scales[:2], 40)
    with pytest.raises(ValueError):
        P.Int8Linear(lin.codes.float(), lin.scales, 40)
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        lin(x, offsets=off, out=torch.zeros((4, 7), device="cuda"))
    assert lin(x[:0], offsets=off).shape == (0, 8)


@pytest.mark.parametrize("t", list(TYPES))
def test_narrow_layers_of_every_width(t):
    # layers of up to 256 channels, rows from one element to past what their kernel holds, with and without experts
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(11)
    for k in (1, 2, 3, 4, 5, 7, 8, 9, 63, 100, 128, 129, 255, 256, 257, 500, 512, 513, 700, 768, 770, 1024, 1027, 1280,
              1401, 1536, 1699, 1792, 1793, 2047, 2048, 2049, 2177):
        m, n, G = 75, (50, 256, 33, 241)[k % 4], 3
        x = torch.from_numpy(rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))).to(TYPES[t]).cuda()
        x[20] = 0
        x[21, k - 1] = float("nan")
        x[22, 0] = float("-inf")
        qx, sx = ox.codes(x.cpu().double().numpy())
        e = rng.integers(-1, G, (m, 1)).astype(np.int32)
        off, rows, _ = ox.plan(e, G)
        r = P.Route(torch.from_numpy(e).cuda(), G)
        qw, sw, b = _layer(rng, G, n, k)
        lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
        tok = np.maximum(rows, 0)
        want, mag = ox.product(qx[tok], sx[tok], qw, sw, b, _groups(off, m, G))
        _check(lin(x, route=r, dtype=torch.float32), want, mag, "f32")
        one = P.Int8Linear(lin.codes[1], lin.scales[1], k)
        want, mag = ox.product(qx, sx, qw[1:2], sw[1:2])
        _check(one(x, dtype=torch.float32), want, mag, "f32")


@pytest.mark.parametrize("m,n,k", [(1, 20, 300), (5, 40000, 130), (8, 3000, 2048), (9, 3000, 2048), (16, 9000, 700),
                                   (16, 70000, 64), (3, 64, 5000), (16, 100, 8200)])
def test_few_rows(m, n, k):
    # every number of wavefronts that share a tile, rows coded inside the kernel and before it
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m + n)
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).cuda()
    qw, sw, b = _layer(rng, 1, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    qx, sx = ox.codes(x.cpu().numpy())
    want, mag = ox.product(qx, sx, qw, sw, b)
    _check(lin(x), want, mag, "f32")
    _check(lin(x, dtype=torch.bfloat16), want, mag, "bf16")


@pytest.mark.parametrize("m,n,k", [(4096, 4096, 1000), (16000, 512, 1600), (2048, 2048, 1000), (3000, 300, 2500)])
@pytest.mark.parametrize("G", [1, 5])
def test_every_tile(m, n, k, G):
    # sizes that take the tiles of 256 x 256, 128 x 128, 128 x 64 and 64 x 64, for one layer and for experts of
    # uneven numbers of rows (one without any) and rows of none
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(m + G)
    qx = rng.integers(-127, 128, (m, k)).astype(np.int8)
    sx = (rng.random(m) * 0.1).astype(np.float32)
    qw, sw, b = _layer(rng, G, n, k)
    off, groups = None, None
    if G > 1:
        off = np.array([0, m // 3 + 5, m // 3 + 5, m // 2, m // 2 + 1, m - 7], np.int64)
        groups = _groups(off, m, G)
        off = torch.from_numpy(off.astype(np.int32)).cuda()
    want, mag = ox.product(qx, sx, qw, sw, b, groups)
    for t in ("f32", "bf16"):
        y = torch.full((m, n), 9.0, dtype=TYPES[t], device="cuda")
        P.dpc_matmul_i8(torch.cuda.current_stream(), P.elem_of(y.dtype), m, 1, n, k, G, _padded(qx, P.i8_ld(k)),
                        torch.from_numpy(sx).cuda(), None, off, _padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(),
                        torch.from_numpy(b).cuda(), y, n)
        _check(y, want, mag, t)


@pytest.mark.parametrize("n", [40, 300])
def test_rows_past_32_bits(n):
    # elements and bytes of x past 2^31 and 2^32, in one kernel (n = 40) and by way of the codes
    import paper_2107_02103_amd as P
    m, k = 1400000, 1600
    x = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    pick = torch.tensor([0, 1, m // 2, m - 33, m - 1], device="cuda")
    x[pick] = torch.randn((5, k), generator=g, device="cuda").to(torch.bfloat16)
    rng = np.random.default_rng(3)
    qw, sw, b = _layer(rng, 1, n, k)
    lin = P.Int8Linear(_padded(qw, P.i8_ld(k)), torch.from_numpy(sw).cuda(), k, torch.from_numpy(b).cuda())
    y = lin(x, dtype=torch.bfloat16)
    qx, sx = ox.codes(x[pick].cpu().double().numpy())
    want, mag = ox.product(qx, sx, qw, sw, b)
    _check(y[pick], want, mag, "bf16")
    rest = torch.ones(m, dtype=torch.bool, device="cuda")
    rest[pick] = False
    assert bool((y[rest] == lin.bias[0].to(torch.bfloat16)).all())
