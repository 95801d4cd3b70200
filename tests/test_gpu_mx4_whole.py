"""4-bit values and layers over many rows, every result compared.

Values have one right value.  A product is summed in float32, 128 terms at a time by the
matrix cores, each such sum and its addition to the running one within 2^-23 of the
magnitudes, and the bias added: (K / 128 + 12) 2^-23 of the sum of magnitudes of its own
row and channel, then a rounding of the result."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f64": torch.float64, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f64": 0.0, "f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
MIB192 = 192 << 20


def _values(codes, scales, cols):
    """What codes and scales of rows stand for, in float64."""
    q = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1).long()
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    e = scales.transpose(0, 1).reshape(codes.shape[0], -1).double()
    scale = torch.where(e == 255, float("nan"), torch.exp2(e - 127.0))
    v = torch.cat([table, -table])[q].view(codes.shape[0], -1, 32) * scale[:, :, None]
    return v.view(codes.shape[0], -1)[:, :cols]


@pytest.mark.parametrize("t,K", [("f64", 520), ("f32", 1600), ("f32", 4), ("f16", 4104), ("bf16", 4096), ("bf16", 240), ("bf16", 8)])
@pytest.mark.parametrize("gap", [0, 1])
def test_values_on_both_sides_of_192_mib(t, K, gap):
    """Results of that size and more are written past the caches, with and without a gap of 16 bytes behind each row."""
    import paper_2107_02103_amd as P
    es = torch.empty((), dtype=TYPES[t]).element_size()
    n, ld = MIB192 // (K * es), K + gap * (16 // es)
    g = torch.Generator("cuda").manual_seed(K)
    blocks = 8 * (P.mx4_ld(K) // 256)
    for rows in (n - 1, n, n + 1):
        codes = torch.randint(0, 256, (rows, P.mx4_ld(K) // 2), dtype=torch.uint8, device="cuda", generator=g)
        scales = torch.randint(112, 140, (blocks // 8, rows, 8), dtype=torch.uint8, device="cuda", generator=g)
        scales[0, 3::1001, 0] = 255
        buf = torch.full((rows, ld), 7.0, dtype=TYPES[t], device="cuda")
        P.Mx4Rows(codes, scales, K).values(TYPES[t], out=buf[:, :K])
        assert (buf[:, K:] == 7.0).all()
        for a in range(0, rows, 1 << 16):
            want = _values(codes[a:a + (1 << 16)], scales[:, a:a + (1 << 16)], K).to(TYPES[t])
            got = buf[a:a + (1 << 16), :K]
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.5), want.nan_to_num(nan=0.5)), rows


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k,G", [(131109, 250, 1030, 1), (131072, 33, 1024, 1), (131105, 256, 1024, 3), (66000, 17, 2049, 2)])
def test_every_row_of_narrow_layers(t, m, n, k, G):
    """Rows that are coded and multiplied in one kernel."""
    import paper_2107_02103_amd as P
    g = torch.Generator("cuda").manual_seed(m + n)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g, dtype=torch.float64)
    lin = P.Mx4Linear.from_weight(normal(G, n, k) * torch.exp(normal(G, n, 1)), normal(G, n))
    x = torch.empty(m, k + 3, dtype=TYPES[t], device="cuda")[:, :k]
    x.copy_(normal(m, k) * torch.exp(0.5 * normal(m, 1)) / (64 if t == "f16" else 1))
    x[7] = 0.0
    x[m - 2, k - 1] = float("inf")
    route, token, off = None, torch.arange(m, device="cuda"), [0, m]
    if G > 1:
        route = P.Route(torch.randint(-1, G, (m, 1), dtype=torch.int32, device="cuda", generator=g), G)
        token, off = route.rows.clamp(min=0).long(), route.offsets.tolist()
    w, bias, coded = lin.weight(torch.float64), lin.bias.double(), P.Mx4Rows.from_rows(x)
    for ty in dict.fromkeys((t, "f32", "f64")):
        out = torch.full((m, n + 1), 9.0, dtype=TYPES[ty], device="cuda")
        lin(x, route=route, dtype=TYPES[ty], out=out[:, :n])
        assert (out[:, n] == 9.0).all() and not out[off[-1]:, :n].any()
        for e in range(G):
            wt = w[e].t().contiguous()
            size = wt.abs()
            for a in range(off[e], off[e + 1], 1 << 15):
                r = slice(a, min(a + (1 << 15), off[e + 1]))
                v = _values(coded.codes[token[r]], coded.scales[:, token[r]], k)
                want, mag = v @ wt + bias[e], v.abs() @ size + bias[e].abs()
                got = out[r, :n].double()
                nan = want.isnan()
                assert torch.equal(got.isnan(), nan)
                bound = 1.001 * STEP[ty] * want.abs() + (k / 128 + 12) * 2.0 ** -23 * mag + LEAST[ty]
                bad = ~nan & ~((got - want).abs() <= bound)
                assert not bad.any(), (ty, e, a, bad.nonzero()[:4], got[bad][:4], want[bad][:4])
