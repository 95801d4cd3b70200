"""Lookups and gradients whose every result has one right value, or one within float64's
roundings of it.

The gradient's sums, and their product with the scale, are float64 arithmetic, rounded
once to the result's type.  A sum of L terms in any order is within (L - 1) 2^-53 of the
sum of their magnitudes, here and in the comparison; the scale adds a rounding on each
side: 2 (L + 1) 2^-53 of the magnitudes and half a step of the result."""
import numpy as np
import pytest

import oracle.gate as og

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f64": 0.0, "f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # half the least number
MIB192 = 192 << 20


def _runs(rng, n, longest):
    """Ids of n tokens in random order, with 1 to `longest` tokens each."""
    lengths = []
    while sum(lengths) < n:
        lengths.append(int(np.exp(rng.uniform(0, np.log(longest)))))
    ids = np.repeat(np.arange(len(lengths)), lengths)[:n].astype(np.int32)
    return ids[rng.permutation(n)], int(ids.max()) + 1


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,longest,W", [(50, 7, 40), (3000, 40, 5), (3000, 40, 240), (20000, 600, 33), (60000, 9000, 12),
                                         (60000, 60000, 3)])
def test_sums_are_float64(t, n, longest, W):
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n + W)
    ids, V = _runs(rng, n, longest)
    ids[rng.random(n) < 0.03] = -1
    dy = torch.from_numpy(rng.standard_normal((n, W)) * np.exp(2 * rng.standard_normal((n, 1)))).cuda().to(TYPES[t])
    plain, dids = dy.cpu().double().numpy(), torch.from_numpy(ids).cuda()
    most = np.bincount(ids[ids >= 0]).max()
    for td in dict.fromkeys((t, "f32")):
        want, mag = og.lookup_backward(ids, plain, V, 0.3)
        got = P.Embedding.gradient(dids, dy, V, 0.3, TYPES[td]).cpu().double().numpy()
        off = 2 * (most + 1) * 2.0 ** -53 * mag
        bound = off + STEP[td] * (np.abs(want) + off) + LEAST[td]
        assert (np.abs(got - want) <= bound).all(), (td, (np.abs(got - want) / bound).max())


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,longest,W", [(60, 12, 9), (60, 12, 64), (3000, 40, 3), (20000, 600, 240), (40000, 9000, 16),
                                         (60000, 60000, 5)])
def test_small_terms_survive_large_ones_that_cancel(t, n, longest, W):
    """Terms of +-2^30 (float16 2^15) that add to nothing, among ones of 2^-6 to 1: sums are below 2^46 in units of 2^-6,
    exact in float64 in every order, and lost in float32."""
    import paper_2107_02103_amd as P
    rng = np.random.default_rng(n * 3 + W)
    ids, V = _runs(rng, n, longest)
    dy = rng.integers(-64, 65, (n, W)) * 2.0 ** -6
    big = 2.0 ** (15 if t == "f16" else 30)
    for v in range(V):                              # the second and third of every four tokens of an id
        at = np.flatnonzero(ids == v) if V < 500 else None
        if at is None:
            break
        dy[at[1::4][:len(at[2::4])]], dy[at[2::4]] = big, -big
    if V >= 500:
        order = np.argsort(ids, kind="stable")
        rank = np.arange(n) - np.searchsorted(ids[order], ids[order])
        count = np.bincount(ids, minlength=V)[ids[order]]
        dy[order[(rank % 4 == 1) & (rank + 1 < count)]] = big
        dy[order[rank % 4 == 2]] = -big
    x = torch.from_numpy(dy).cuda().to(TYPES[t])
    np.testing.assert_array_equal(x.cpu().double().numpy(), dy)
    want, _ = og.lookup_backward(ids, dy, V)
    assert np.abs(want).max() < 2.0 ** 17           # nothing large is left: 24 bits hold it
    td = TYPES["f64" if t == "f64" else "f32"]
    got = P.Embedding.gradient(torch.from_numpy(ids).cuda(), x, V, dtype=td)
    np.testing.assert_array_equal(got.cpu().double().numpy(), want)


@pytest.mark.parametrize("W", [1, 8, 70])
def test_a_sum_is_rounded_once(W):
    """Sums a little above and below the middle of two neighbours of the result's type, by less than float32 shows: through
    float32 they would be taken for the middle."""
    import paper_2107_02103_amd as P
    for t, half in (("bf16", 2.0 ** -8), ("f16", 2.0 ** -11)):
        tiny = 2.0 ** -30 if t == "bf16" else 2.0 ** -24          # the least number of float16
        # 1 + half is a tie that goes to 1, 1 + 3 half one that goes to 1 + 4 half
        rows = np.array([[1, half, tiny], [1, half, -tiny], [1, half, 0], [1, 3 * half, -tiny], [1, 3 * half, tiny],
                         [1, 3 * half, 0]])
        sure = np.array([1 + 2 * half, 1, 1, 1 + 2 * half, 1 + 4 * half, 1 + 4 * half])
        if t == "f16":
            # float32 holds 1 + 2^-11 + 2^-24 itself only up to its own half step, which goes to the even one, the tie
            assert np.float32(1 + half + tiny) == np.float32(1 + half)
        ids = torch.arange(6, dtype=torch.int32, device="cuda").repeat_interleave(3)
        dy = torch.from_numpy(rows.reshape(-1, 1).repeat(W, 1)).cuda().to(TYPES[t])
        np.testing.assert_array_equal(dy.cpu().double().numpy(), rows.reshape(-1, 1).repeat(W, 1))
        got = P.Embedding.gradient(ids, dy, 6).cpu().double().numpy()
        np.testing.assert_array_equal(got, sure[:, None].repeat(W, 1))


def _lookup(table, ids, scale):
    """The same in torch: a product in float32 (float64), rounded to the table's type."""
    acc = torch.float64 if table.dtype == torch.float64 else torch.float32
    live = (ids >= 0) & (ids < table.shape[0])
    y = (table.to(acc) * torch.tensor(scale, dtype=acc, device="cuda")).to(table.dtype)[torch.where(live, ids, 0).long()]
    return y.masked_fill_(~live[:, None], 0.0)


def _table(g, V, W, t):
    return torch.randn(V, W, device="cuda", generator=g, dtype=torch.float64).to(TYPES[t])


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,V,W", [(1, 3, 240), (5, 2, 16), (257, 3, 240), (1000, 3, 1600), (129, 3000, 4104), (4099, 40000, 64),
                                   (70001, 5, 8), (33333, 70, 1032), (3, 1, 65536)])
def test_lookup_without_gaps(t, n, V, W):
    """Results that the call allocates: one array of chunks of 16 bytes, whose last workgroup is not full."""
    import paper_2107_02103_amd as P
    g = torch.Generator("cuda").manual_seed(n + W)
    table = _table(g, V, W, t)
    ids = torch.randint(-1, V + 1, (n,), dtype=torch.int32, device="cuda", generator=g)
    ids[-1] = V - 1
    for scale in (1.0, 0.3, -64.0):
        y = P.Embedding(table, scale)(ids)
        assert y.is_contiguous() and torch.equal(y, _lookup(table, ids, scale))
    wide = _table(g, V, W + 3, t)[:, :W]            # rows at addresses that only their elements divide
    assert torch.equal(P.Embedding(wide, 0.3)(ids), _lookup(wide, ids, 0.3))


@pytest.mark.parametrize("t,W", [("f64", 120), ("f32", 240), ("f16", 480), ("bf16", 4096), ("f32", 4)])
@pytest.mark.parametrize("gap", [0, 1])
def test_lookup_on_both_sides_of_192_mib(t, W, gap):
    """Results of that size and more are written past the caches, with and without a gap of 16 bytes behind each row."""
    import paper_2107_02103_amd as P
    es = torch.empty((), dtype=TYPES[t]).element_size()
    n, ld = MIB192 // (W * es), W + gap * (16 // es)
    g = torch.Generator("cuda").manual_seed(W)
    table = _table(g, 37, W, t)
    for rows in (n - 1, n, n + 1, n + 1003):
        ids = torch.randint(-1, 38, (rows,), dtype=torch.int32, device="cuda", generator=g)
        buf = torch.full((rows, ld), 6.0, dtype=TYPES[t], device="cuda")
        P.Embedding(table, 0.3)(ids, out=buf[:, :W])
        assert torch.equal(buf[:, :W], _lookup(table, ids, 0.3)), rows
        assert (buf[:, W:] == 6.0).all()
