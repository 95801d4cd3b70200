"""A mixture of nets in 4 bits, run as a user runs it: vectors of species to scores,
choice, routing, the experts' layers, back to the atoms; against the same from the
plain definitions in 64 bits, eagerly, captured and on a stream of its own."""
import numpy as np
import pytest

import oracle.experts as ox
import oracle.gate as og
import oracle.mx4 as om

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Mixture:
    def __init__(self, table, vectors, bias, W, b, topk, groups):
        import paper_2107_02103_amd as P
        self.P, self.E = P, W.shape[0]
        self.scores, self.vectors = P.Embedding(table), P.Embedding(vectors, 0.5)
        self.gate = P.Gate(self.E, topk, "sigmoid", groups, groups // 2, 2, bias, renormalise=True)
        self.layer = P.Mx4Linear.from_weight(W, b)

    def __call__(self, x, species):
        h = x + self.vectors(species)
        expert, weight = self.gate(self.scores(species))
        route = self.P.Route(expert, self.E)
        return route.combine(self.layer(h, route=route), weight), expert, weight, h


@pytest.mark.parametrize("n,K,N,E,groups,topk", [(1, 96, 40, 8, 4, 2), (9, 300, 64, 16, 4, 3), (400, 256, 130, 8, 2, 2),
                                                 (3000, 513, 64, 4, 2, 1)])
def test_a_mixture_of_layers(n, K, N, E, groups, topk):
    rng = np.random.default_rng(n)
    species, S = rng.integers(-1, 5, n).astype(np.int32), 5
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    table, vectors = rng.standard_normal((S, E)).astype(np.float32), rng.standard_normal((S, K)).astype(np.float32)
    table[1, 0] = -np.inf                                     # an expert that is closed to a species
    bias, b = (0.1 * rng.standard_normal(E)).astype(np.float32), rng.standard_normal((E, N)).astype(np.float32)
    W, x = (rng.standard_normal((E, N, K)) / np.sqrt(K)).astype(np.float32), rng.standard_normal((n, K)).astype(np.float32)
    m = Mixture(dev(table), dev(vectors), dev(bias), dev(W), dev(b), topk, groups)
    dx, ds = dev(x), dev(species)
    y, expert, weight, h = m(dx, ds)
    # padding atoms (species -1) have scores of 0 everywhere and are routed like any other row
    we, ww = og.choose(og.lookup(table, species), topk, "sigmoid", bias, groups, groups // 2, 2, True)
    np.testing.assert_array_equal(expert.cpu().numpy(), we)
    plain = om.values(*om.quantise(h.cpu().double().numpy()))[:, :K]
    values = [om.values(*om.quantise(w))[:, :K] for w in W]
    off, rows, pos = ox.plan(we, E)
    out, mag = np.zeros((n * topk, N)), np.zeros((n * topk, N))
    for e in range(E):
        r = slice(off[e], off[e + 1])
        out[r], mag[r] = om.product(plain[rows[r] // topk], values[e], b[e])
    want, _ = ox.combine(out, pos, ww)
    size, _ = ox.combine(mag, pos, np.abs(ww))
    # each product within (K / 128 + 12) 2^-23 of its magnitudes, weights and products rounded, topk of them summed
    assert (np.abs(y.cpu().double().numpy() - want) <= (K / 128 + 16 + topk) * 2.0 ** -23 * size).all()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2 = m(dx, ds)[0]
    s.synchronize()
    assert torch.equal(y, y2)
    bx, bs, graph = dx.clone(), ds.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = m(bx, bs)[:3]
    for i in range(3):
        bx.copy_(torch.randn(n, K, device="cuda"))
        bs.copy_(dev(rng.integers(-1, S, n).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        for a, b_ in zip(captured, m(bx, bs)[:3]):
            assert torch.equal(a, b_)


def test_gradients_of_the_mixture_against_differences():
    """dE/dtable and dE/dvectors of E = sum(y^2) / 2 with the layers as values that their codes stand for, in float64:
    the straight products' gradient, which a training step with 4-bit weights takes."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(7)
    n, K, N, E, S, topk = 60, 40, 6, 4, 3, 2
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    species = dev(rng.integers(-1, S, n).astype(np.int32))
    table, vectors, x = dev(rng.standard_normal((S, E))), dev(rng.standard_normal((S, K))), dev(rng.standard_normal((n, K)))
    W = P.Mx4Linear.from_weight(dev(rng.standard_normal((E, N, K)))).weight(torch.float64)

    def run(table, vectors, grad=False):
        scores, vec = P.Embedding(table), P.Embedding(vectors, 0.5)
        gate = P.Gate(E, topk, "softmax", renormalise=True)
        z, h = scores(species), x + vec(species)
        expert, weight = gate(z)
        route = P.Route(expert, E)
        rows, off = route.gather(h), route.offsets.tolist()
        out = torch.zeros(n * topk, N, dtype=torch.float64, device="cuda")
        for e in range(E):
            out[off[e]:off[e + 1]] = rows[off[e]:off[e + 1]] @ W[e].t().contiguous()
        y = route.combine(out, weight)
        if not grad:
            return float((y * y).sum()) / 2, expert
        dout, dw = route.combine_backward(out, y, weight)
        drows = torch.zeros_like(rows)
        for e in range(E):
            drows[off[e]:off[e + 1]] = dout[off[e]:off[e + 1]] @ W[e].contiguous()
        dh = route.combine(drows)
        return scores.backward(species, gate.backward(z, expert, dw)), vec.backward(species, dh)

    (dt, dv), (base, chosen) = run(table, vectors, True), run(table, vectors)
    for which, t, d in (("table", table, dt), ("vectors", vectors, dv)):
        for i in rng.choice(t.numel(), min(12, t.numel()), replace=False):
            h, up, dn = 1e-5, t.clone(), t.clone()
            up.view(-1)[i] += h
            dn.view(-1)[i] -= h
            (a, ea), (b, eb) = (run(u, vectors) if which == "table" else run(table, u) for u in (up, dn))
            assert torch.equal(ea, chosen) and torch.equal(eb, chosen)
            # third derivatives under 100 E times h^2, roundings of E of 2^-50 / h
            assert abs((a - b) / (2 * h) - float(d.view(-1)[i])) < 100 * base * h * h + base * 2.0 ** -50 / h
