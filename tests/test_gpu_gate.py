"""The choice of experts and its gradient on the GPU against the plain ones in 64
bits.

Choices are made in float64 on both sides and are equal (equal scores are equal on
both, and go to the lower expert).  A weight is off by its own rounding (2^-24, for
float64 logits 2^-53) and the float64 arithmetic before it: exponentials within an
ulp or two, a sum of E terms and one of topk, a few products: 2 (E + 64) 2^-53 covers
both sides.  The gradient is float32 arithmetic: exponentials of arguments rounded
to 2^-24 of their size, sums of E and of topk terms, a few products; then one
rounding to the type of the logits."""
import numpy as np
import pytest

import oracle.gate as og

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f64": 2.0 ** -1000, "f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}


def _case(rng, n, E, t, closed, pad=0, shift=0, grid=None):
    """Logits on the GPU in rows apart by E + pad from an address that only the element divides, and as float64."""
    z = 2.0 * rng.standard_normal((n, E)) + rng.standard_normal(E)
    if grid:
        z = np.round(z * grid) / grid                       # many equal scores
    if closed:
        z[rng.random((n, E)) < closed] = -np.inf
        z[n // 2] = -np.inf
    buf = torch.full((shift + n * (E + pad) + 8,), 77.0, dtype=TYPES[t], device="cuda")
    x = buf[shift:shift + n * (E + pad)].view(n, E + pad)[:, :E]
    x.copy_(torch.from_numpy(z))
    return x, x.cpu().double().numpy()


def _check_weights(got, want, E, t):
    got = got.cpu().double().numpy()
    unit = STEP["f64" if t == "f64" else "f32"]
    bound = np.abs(want) * (1.001 * unit + 2 * (E + 64) * 2.0 ** -53) + (0 if t == "f64" else 2.0 ** -149)
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()


SHAPES = [
    (1, 1, 1, 1, 1, 1), (5, 2, 2, 1, 1, 1), (70, 3, 2, 1, 1, 1), (1000, 3, 1, 1, 1, 1), (33, 4, 4, 2, 1, 2),
    (65, 5, 3, 1, 1, 1), (64, 8, 2, 4, 2, 1), (100, 9, 4, 3, 2, 2), (31, 16, 16, 1, 1, 1), (40, 17, 5, 1, 1, 1),
    (50, 32, 4, 4, 2, 2), (21, 33, 8, 11, 3, 1), (257, 64, 6, 8, 3, 2), (19, 100, 10, 5, 5, 2), (30, 127, 7, 1, 1, 1),
    (30, 128, 8, 8, 4, 2), (9, 160, 64, 1, 1, 1), (300, 256, 8, 8, 4, 2), (11, 257, 3, 1, 1, 1), (7, 384, 6, 64, 9, 2),
    (6, 512, 8, 16, 1, 2), (6, 513, 8, 27, 20, 2), (4, 1000, 64, 8, 8, 1), (5, 1024, 16, 64, 64, 2), (3, 1024, 64, 1, 1, 1)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,E,k,groups,keep,best", SHAPES)
def test_choice(t, n, E, k, groups, keep, best):
    import paper_2107_02103_amd as P
    k = min(k, keep * (E // groups))
    for v, (kind, biased, renorm, closed, grid) in enumerate((
            ("softmax", False, True, 0.0, None), ("sigmoid", True, True, 0.3, None), ("softmax", True, False, 0.6, 4),
            ("sigmoid", False, False, 0.0, 2))):
        rng = np.random.default_rng(100 * E + n + v)
        z, plain = _case(rng, n, E, t, closed, pad=v, shift=v % 2, grid=grid)
        bias = rng.standard_normal(E).astype(np.float32) * 0.2 if biased else None
        if kind == "sigmoid" and grid:
            # the sums of s(z) and s(-z) are 1 for every z: pairs of groups that only rounding tells apart
            z.abs_()
            plain = np.abs(plain)
        gate = P.Gate(E, k, kind, groups, keep, best, None if bias is None else torch.from_numpy(bias).cuda(), renorm, 2.5)
        e, w = gate(z)
        assert e.dtype == torch.int32 and w.dtype == (torch.float64 if t == "f64" else torch.float32)
        we, ww = og.choose(plain, k, kind, bias, groups, keep, best, renorm, 2.5)
        np.testing.assert_array_equal(e.cpu().numpy(), we)
        _check_weights(w, ww, E, t)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,E,k", [(s[0], s[1], min(s[2], s[1])) for s in SHAPES])
def test_gradient(t, n, E, k):
    import paper_2107_02103_amd as P
    for v, (kind, renorm, closed) in enumerate((("softmax", True, 0.3), ("sigmoid", True, 0.0), ("softmax", False, 0.0),
                                                ("sigmoid", False, 0.5))):
        rng = np.random.default_rng(100 * E + n + v)
        z, plain = _case(rng, n, E, t, closed, pad=v, shift=v % 2)
        e, _ = og.choose(plain, k, kind)
        d = rng.standard_normal((n, k))
        if n > 4:
            e[1] = e[1, 0]                                  # the same expert twice
            e[2, -1], d[2, -1] = -1, np.nan                 # dropped: what stands there does not count
            e[3, 0], d[3, 0] = E, np.inf
        wt = torch.float64 if t == "f64" else torch.float32
        dw = torch.from_numpy(d).to(wt).cuda()
        out = torch.full((n, E + 3), 55.0, dtype=TYPES[t], device="cuda")
        P.Gate(E, k, kind, renormalise=renorm, scale=0.7).backward(z, torch.from_numpy(e.astype(np.int32)).cuda(), dw,
                                                                    out=out[:, :E])
        assert (out[:, E:] == 55.0).all()
        got = out[:, :E].cpu().double().numpy()
        want, mag = og.choose_backward(plain, e, dw.cpu().double().numpy(), kind, renorm, 0.7)
        unit = STEP["f64" if t == "f64" else "f32"]
        size = np.abs(np.where(np.isfinite(plain), plain, 0)).max()
        bound = 1.001 * STEP[t] * np.abs(want) + (E + k + 64 + 2 * size) * unit * mag + LEAST[t]
        assert (np.abs(got - want) <= bound).all(), (kind, renorm, np.abs(got - want).max())


@pytest.mark.parametrize("E,k,groups,keep,best", [(3, 2, 1, 1, 1), (12, 4, 4, 2, 2), (40, 6, 1, 1, 1), (100, 8, 10, 3, 2),
                                                  (256, 8, 8, 4, 2), (256, 40, 1, 1, 1), (1000, 8, 8, 3, 1)])
def test_scores_that_float32_cannot_tell_apart(E, k, groups, keep, best):
    """Scores 10^-7 apart, as near as float32 may be off, and sums of two that differ in second order, by 10^-14: still a
    hundred roundings of float64."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(E + k)
    n = 200
    z = (1.0 + 2.0 ** -21 * rng.integers(0, 40, (n, E))).astype(np.float32)
    z[1::3] += (rng.integers(-2, 2, (len(z[1::3]), E)) * 0.25).astype(np.float32)
    bias = (rng.integers(0, 3, E) * 2.0 ** -20).astype(np.float32)
    for kind, b in (("sigmoid", bias), ("softmax", bias), ("sigmoid", None), ("softmax", None)):
        e, w = P.Gate(E, k, kind, groups, keep, best, None if b is None else torch.from_numpy(b).cuda(), True)(
            torch.from_numpy(z).cuda())
        we, ww = og.choose(z, k, kind, b, groups, keep, best, True)
        np.testing.assert_array_equal(e.cpu().numpy(), we)
        _check_weights(w, ww, E, "f32")


def test_equal_scores_of_every_expert():
    """As a gate of zeros gives them: the lowest experts (of the lowest groups)."""
    import paper_2107_02103_amd as P
    for E, k, groups, keep in ((3, 2, 1, 1), (64, 8, 8, 2), (256, 8, 1, 1), (700, 64, 7, 3)):
        z = torch.full((37, E), -0.0, device="cuda")
        z[:, ::2] = 0.0
        for t in (torch.float32, torch.bfloat16, torch.float64):
            for kind in ("softmax", "sigmoid"):
                e, w = P.Gate(E, k, kind, groups, keep, 2, renormalise=True)(z.to(t))
                assert (e.cpu() == torch.arange(k)).all() and (w * k - 1).abs().max() < 1e-6


def test_rows_with_nan_and_infinity():
    import paper_2107_02103_amd as P
    for E, k in ((3, 2), (20, 4), (200, 8)):
        z = torch.randn(6, E, device="cuda")
        z[1, E // 2] = float("nan")
        z[2, 0] = float("inf")
        z[3] = -float("inf")
        z[4, 1:] = -float("inf")
        z[5] = torch.finfo(torch.float32).min            # the lowest value closes nothing
        for kind in ("softmax", "sigmoid"):
            bias = torch.full((E,), 0.25, device="cuda")
            for gate in (P.Gate(E, k, kind, renormalise=True), P.Gate(E, k, kind, bias=bias)):
                e, w = gate(z)
                e, w = e.cpu(), w.cpu()
                assert w[1].isnan().all() and e[1].tolist() == list(range(k))
                if kind == "softmax":
                    assert w[2].isnan().all() and e[2].tolist() == list(range(k))
                else:
                    assert w[2].isfinite().all() and e[2, 0] == 0
                assert (e[3] == -1).all() and (w[3] == 0).all()
                assert e[4, 0] == 0 and (e[4, 1:] == -1).all() and (w[4, 1:] == 0).all()
                assert e[5].tolist() == list(range(k)) and w[5].isfinite().all()
                assert w[0].isfinite().all()
        bias = torch.zeros(E, device="cuda")
        bias[1] = -float("inf")
        e, w = P.Gate(E, k, "softmax", bias=bias)(z)
        assert not (e[0] == 1).any() and w[0].isfinite().all()
        bias[1] = float("nan")
        e, w = P.Gate(E, k, "softmax", bias=bias)(z)
        assert w.isnan().all()


def test_no_tokens_streams_and_graphs():
    import paper_2107_02103_amd as P
    gate = P.Gate(64, 4, "sigmoid", 8, 4, 2, torch.zeros(64, device="cuda"), True)
    e, w = gate(torch.empty(0, 64, device="cuda"))
    assert e.shape == w.shape == (0, 4)
    assert gate.backward(torch.empty(0, 64, device="cuda"), e, w).shape == (0, 64)
    z = torch.randn(500, 64, device="cuda")
    want = gate(z)
    dw = torch.randn(500, 4, device="cuda")
    dz = gate.backward(z, want[0], dw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = gate(z, stream=s)
    dgot = gate.backward(z, got[0], dw, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(dgot, dz)
    buf = z.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ge, gw = gate(buf)
        gd = gate.backward(buf, ge, dw)
    for i in range(3):
        buf.copy_(torch.randn(500, 64, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        e, w = gate(buf)
        assert torch.equal(ge, e) and torch.equal(gw, w) and torch.equal(gd, gate.backward(buf, e, dw))


def test_chain_with_route_and_gradient_of_a_mixture():
    """Vectors of species to logits, choice, routing and back: energies of a mixture and the gradient of the table
    against the same in 64 bits and against differences."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(5)
    n, species, E, k, W = 400, 3, 6, 2, 24
    ids = torch.from_numpy(rng.integers(-1, species, n).astype(np.int32)).cuda()
    table = torch.from_numpy(rng.standard_normal((species, E))).cuda()
    x = torch.from_numpy(rng.standard_normal((n, W))).cuda()
    nets = torch.from_numpy(rng.standard_normal((E, W))).cuda()
    emb, gate = P.Embedding(table, 2.0), P.Gate(E, k, "softmax", renormalise=True)

    def energy(table, grad=False):
        emb = P.Embedding(table, 2.0)
        z = emb(ids)
        expert, weight = gate(z)
        route = P.Route(expert, E)
        rows = route.gather(x)
        who = expert.reshape(-1)[route.rows.clamp(min=0).long()].long()
        e_rows = torch.tanh((rows * nets[who]).sum(1, keepdim=True))
        y = route.combine(e_rows, weight)
        if not grad:
            return y.sum().item(), expert
        _, dw = route.combine_backward(e_rows, torch.ones_like(y), weight, need_rows=False)
        return emb.backward(ids, gate.backward(z, expert, dw))

    d = energy(table, True).cpu().numpy()
    base = energy(table)[1]
    for v in range(species):
        for e in range(E):
            h, up, dn = 1e-5, table.clone(), table.clone()
            up[v, e] += h
            dn[v, e] -= h
            (a, ea), (b, eb) = energy(up), energy(dn)
            assert torch.equal(ea, base) and torch.equal(eb, base)
            # third derivatives of order 10 n times h^2, roundings n 2^-52 / h
            assert abs((a - b) / (2 * h) - d[v, e]) < 10 * n * h * h + n * 2.0 ** -50 / h


@pytest.mark.parametrize("E,groups,k", [(4, 4, 4), (8, 8, 8), (16, 16, 16), (32, 32, 32), (64, 64, 64), (48, 16, 30)])
def test_as_many_groups_as_experts(E, groups, k):
    """The most LDS that a wavefront takes, and groups of one expert."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(E)
    z = rng.standard_normal((130, E)).astype(np.float32)
    z[5::7] = -np.inf
    bias = rng.standard_normal(E).astype(np.float32)
    for keep in (groups, max(1, groups // 2)):
        kk = min(k, keep * (E // groups))
        for t in (torch.float32, torch.float64):
            e, w = P.Gate(E, kk, "softmax", groups, keep, 2, torch.from_numpy(bias).cuda())(torch.from_numpy(z).cuda().to(t))
            we, ww = og.choose(z, kk, "softmax", bias, groups, keep, 2)
            np.testing.assert_array_equal(e.cpu().numpy(), we)
            _check_weights(w, ww, E, "f64" if t == torch.float64 else "f32")


def test_tokens_past_32_bits():
    """Rows of logits that start behind 2^31 elements, read and written."""
    import paper_2107_02103_amd as P
    far = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(far, (3, 64), ((1 << 30) + 512, 1))
    z.copy_(torch.randn(3, 64))
    gate = P.Gate(64, 4, "softmax")
    e, w = gate(z)
    near = z.clone()
    e2, w2 = gate(near)
    assert torch.equal(e, e2) and torch.equal(w, w2)
    dw = torch.randn(3, 4, device="cuda")
    out = torch.as_strided(far, (3, 64), ((1 << 30) + 512, 1), 128)
    gate.backward(z, e, dw, out=out)
    assert torch.equal(out, gate.backward(near, e, dw))


def test_many_tokens():
    """More than one dimension of a launch takes at once, in workgroups of 256 tokens: checked by what is known."""
    import paper_2107_02103_amd as P
    n = (1 << 30) + 300
    z = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")
    z[-1] = -float("inf")
    with pytest.raises(P.DpcError):
        P.Gate(1, 1)(z)
    z = z[-(1 << 30):]
    e, w = P.Gate(1, 1, "sigmoid", scale=4.0)(z)
    assert e[-1] == -1 and w[-1] == 0 and not e[:-1].any() and bool((w[:-1] == 2.0).all())


@pytest.mark.parametrize("t", ["f64", "f32", "bf16"])
@pytest.mark.parametrize("E,k", [(3, 2), (7, 3), (40, 6), (200, 8), (900, 8)])
def test_gradient_where_scores_are_tiny(t, E, k):
    """Chosen experts (a bias can choose any) whose scores are e^-90 to e^-600, below float32's smallest number: their
    shares, and the gradient, are of order 1 all the same; and scores within e^-30 of 1."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(E)
    n = 41
    far = rng.choice([0.0, 60.0, 90.0, 150.0, 600.0], n)[:, None]
    base = rng.standard_normal((n, E))
    e = np.stack([rng.permutation(E)[:k] for _ in range(n)])
    for kind, z in (("sigmoid", base - far), ("sigmoid", base + np.minimum(far, 30.0)), ("softmax", base.copy())):
        if kind == "softmax":
            for i in range(n):
                z[i, e[i]] -= far[i]                        # the others hold nearly all of the sum
        z[5], z[6] = -2000.0, -np.inf                       # no share: the sum is 0 in float64
        if kind == "softmax" and E > k:
            z[5, np.setdiff1d(np.arange(E), e[5])] = 0.0
        x = torch.from_numpy(z).to(TYPES[t]).cuda()
        plain = x.cpu().double().numpy()
        wt = torch.float64 if t == "f64" else torch.float32
        dw = torch.from_numpy(rng.standard_normal((n, k))).to(wt).cuda()
        for renorm in (True, False):
            got = P.Gate(E, k, kind, renormalise=renorm).backward(x, torch.from_numpy(e.astype(np.int32)).cuda(), dw)
            got = got.cpu().double().numpy()
            want, mag = og.choose_backward(plain, e, dw.cpu().double().numpy(), kind, renorm)
            unit = STEP["f64" if t == "f64" else "f32"]
            size = np.abs(np.where(np.isfinite(plain), plain, 0)).max(1, keepdims=True)
            bound = 1.001 * STEP[t] * np.abs(want) + (E + k + 64 + 2 * size) * unit * mag + LEAST[t]
            assert (np.abs(got - want) <= bound).all(), (kind, renorm, np.abs(got - want).max())
            if renorm and E > 3:
                assert np.abs(want).max() > 1e-2


def test_gradient_of_rows_with_nan_and_infinity():
    """NaN at all open experts where the weights are NaN, zeros where there is none."""
    import paper_2107_02103_amd as P
    for E, k in ((3, 2), (20, 4), (200, 8)):
        z = torch.randn(5, E, device="cuda")
        z[:, 1] = -float("inf")
        z[1, E // 2 + 1] = float("nan")
        z[2, 0] = float("inf")
        z[3] = -float("inf")
        e = torch.tensor([[0] + list(range(2, k + 1))] * 5, dtype=torch.int32, device="cuda")
        dw = torch.randn(5, k, device="cuda")
        for kind in ("softmax", "sigmoid"):
            for renorm in (True, False):
                d = P.Gate(E, k, kind, renormalise=renorm).backward(z, e, dw)
                assert not d[:, 1].any() and not d[3].any()
                rest = torch.arange(E, device="cuda") != 1
                assert d[1, rest].isnan().all()
                assert d[2, rest].isnan().all() if kind == "softmax" else d[2].isfinite().all()
                assert d[0].isfinite().all() and d[4].isfinite().all()
