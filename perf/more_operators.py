"""Timed cases of the operators around the routing: the choice of experts, learned vectors of ids, and layers in
microscaled 4-bit floating point.

Seven paths:

* "gate"       experts and weights of each token from its scores: softmax or sigmoid, a bias for balance, groups,
               the largest k, renormalised;
* "gate_bwd"   the gradient of the weights in the scores;
* "embed"      vectors of ids, scaled;
* "embed_bwd"  their gradient, summed id by id;
* "codes"      rows to 4-bit codes with a power of two for every 32, and the values that these stand for;
* "linear"     a dense layer on such codes of its rows and weights;
* "expert"     the same layer with one set of weights for each expert over routed rows.

Every path has a plain form in elementary torch operations and, with ``own`` set, the calls of the library.  The
plain forms compute in 32 bits; scores that decide a choice and sums over many tokens in 64.  All inputs come from
the seed alone.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK, STEP = 32, 256         # elements that share a scale; rows of codes are padded to a multiple of STEP elements
TINY = 2.0 ** -100            # blocks whose largest magnitude is below this hold zeros
INF = float("inf")


def listed():
    return [
        # one token of a served mixture: latency
        dict(name="gate_one_bf16", path="gate", tokens=1, experts=64, topk=2, score="softmax", groups=1, keep=1, best=1,
             bias=False, renorm=True, scale=1.0, closed=0, dtype="bf16"),
        # a large batch of a mixture that is balanced by a bias and keeps half of its groups
        dict(name="gate_mix_bf16", path="gate", tokens=65536, experts=256, topk=8, score="sigmoid", groups=8, keep=4,
             best=2, bias=True, renorm=True, scale=2.5, closed=0, dtype="bf16"),
        # the atoms of a large box that are mixtures of the two likeliest of three species: gradient of the weights
        dict(name="gate_bwd_alloy_f32", path="gate_bwd", tokens=331776, experts=3, topk=2, score="softmax", groups=1,
             keep=1, best=1, bias=False, renorm=False, scale=1.0, closed=5, dtype="f32"),
        # a vector for the species of each atom of the million-atom workload: bound by what it writes
        dict(name="embed_types_f32", path="embed", tokens=1048576, ids=3, width=240, scale=1.0, dtype="f32", skew=1.0,
             empty=0),
        # the gradient of the species' vectors: sums over a hundred thousand atoms each
        dict(name="embed_bwd_types_f32", path="embed_bwd", tokens=331776, ids=2, width=240, scale=1.0, dtype="f32",
             skew=0.6, empty=0),
        # the gradient of a vocabulary, padded batch: few tokens an id, most ids without any
        dict(name="embed_bwd_vocab_bf16", path="embed_bwd", tokens=16384, ids=65536, width=4096, scale=64.0, dtype="bf16",
             skew=1.0, empty=10),
        # the rows of a large batch to 4 bits, and the values that a check or another layer takes back from them
        dict(name="codes_mix_bf16", path="codes", tokens=32768, inner=4096, dtype="bf16", out="bf16"),
        # first fitting layer of one atom: latency
        dict(name="linear_one_f32", path="linear", tokens=1, inner=1600, outer=240, dtype="f32", out="f32"),
        # a few tokens through a wide layer: every weight is read for 16 rows
        dict(name="linear_few_bf16", path="linear", tokens=16, inner=8192, outer=8192, dtype="bf16", out="bf16"),
        # first fitting layer of the million-atom workload: the descriptors are read once
        dict(name="linear_cu1m_f32", path="linear", tokens=1048576, inner=1600, outer=240, dtype="f32", out="f32"),
        # a serving step of a mixture: few rows, each with weights of its own
        dict(name="expert_few_bf16", path="expert", tokens=8, topk=2, experts=64, inner=2048, outer=2048, dtype="bf16",
             out="bf16", drop=0, skew=0.0),
        # a large batch of a mixture: bound by the products
        dict(name="expert_mix_bf16", path="expert", tokens=16384, topk=2, experts=16, inner=4096, outer=4096,
             dtype="bf16", out="bf16", drop=2, skew=0.5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the same ranges; no more bytes or operations than the largest listed one of its kind."""
    path = rng.choice(["gate", "gate_bwd", "embed", "embed_bwd", "codes", "linear", "expert"])
    kind = path.split("_")[0]
    most = [work(c) for c in listed() if c["path"].split("_")[0] == kind]
    while True:
        c = dict(path=path, dtype=rng.choice(["f32", "f16", "bf16"]))
        if kind == "gate":
            groups = rng.choice([1, 1, 1, 2, 4, 8])
            per = _log(rng, 4, 1024 // groups) if groups > 1 else _log(rng, 1, 1024)
            keep = rng.randint(1, groups)
            score = rng.choice(["softmax", "sigmoid"])
            c.update(tokens=_log(rng, 1, 400000), experts=groups * per, groups=groups, keep=keep, best=rng.choice([1, 2]),
                     topk=min(rng.choice([1, 2, 2, 3, 4, 6, 8, 8, 16]), keep * per), score=score,
                     bias=rng.random() < (0.5 if score == "softmax" else 0.8) or (score == "sigmoid" and groups > 1),
                     renorm=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 2.5]), closed=rng.choice([0, 0, 5, 40]))
        elif kind == "embed":
            c.update(tokens=_log(rng, 1, 1048576), ids=rng.choice([_log(rng, 1, 200000), _log(rng, 1, 128)]),
                     width=rng.choice([_log(rng, 1, 8192), 240, 1600, 8 * (_log(rng, 4, 512) | 1)]),
                     scale=rng.choice([1.0, 64.0, 0.3]), skew=rng.choice([0.0, 0.6, 1.0, 2.0]), empty=rng.choice([0, 0, 10]))
        else:
            sizes = [_log(rng, 1, 8192), 240, 1600, 64 * (_log(rng, 2, 126) | 1)]
            c.update(tokens=_log(rng, 1, 1048576), inner=rng.choice(sizes))
            c["out"] = "f32" if c["dtype"] == "f16" else rng.choice(["f32", c["dtype"]])
            if kind != "codes":
                c.update(outer=rng.choice(sizes))
            if kind == "expert":
                c.update(topk=rng.choice([1, 1, 2, 4]), experts=_log(rng, 1, 128), drop=rng.choice([0, 0, 5]),
                         skew=rng.choice([0.0, 0.5, 2.0]))
        w = work(c)
        if all(w[k] <= max(m[k] for m in most) for k in w):
            return c


def work(case):
    """Inputs read once, outputs written once.  Scores: four operations each (exponential, sum, bias, comparison);
    vectors: one for each element; products: one multiply and one add for each term."""
    n, e = case["tokens"], SIZE[case["dtype"]]
    path = case["path"]
    if path in ("gate", "gate_bwd"):
        E, k = case["experts"], case["topk"]
        moved = n * E * e * (1 if path == "gate" else 2) + 8 * n * k + (4 * E if case["bias"] and path == "gate" else 0)
        return {"bytes": float(moved), "flops": 4.0 * n * E}
    if path == "embed":
        return {"bytes": float(4 * n + (n + min(n, case["ids"])) * case["width"] * e), "flops": 1.0 * n * case["width"]}
    if path == "embed_bwd":
        return {"bytes": float(4 * n + (n + case["ids"]) * case["width"] * e), "flops": 1.0 * n * case["width"]}
    K, o = case["inner"], SIZE[case["out"]]
    if path == "codes":
        return {"bytes": float(n * K * (e + o) + n * -(-K // BLOCK) * 4), "flops": 2.0 * n * K}
    N, rows = case["outer"], n * case.get("topk", 1)
    groups = min(case.get("experts", 1), rows)            # an expert without rows is not read
    return {"bytes": float(n * K * e + groups * N * (K * 17 / 32 + 4) + rows * N * o + (4 * rows if "topk" in case else 0)),
            "flops": 2.0 * rows * N * K}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _logits(case, g):
    """Scores with experts that are liked by all tokens, some closed (-inf) for some tokens; a token in 61 finds all
    of them closed where any are."""
    n, E = case["tokens"], case["experts"]
    z = (_randn(g, n, E) * 1.5 + _randn(g, E)).to(TYPES[case["dtype"]])
    if case["closed"]:
        z[_rand(g, n, E) < case["closed"] / 100.0] = -INF
        z[7::61] = -INF
    return z


def _some(g, n, of, skew, drop):
    """n numbers below ``of``, uneven by ``skew``; -1 in ``drop`` per cent of the places."""
    p = torch.arange(1, of + 1, device=DEV, dtype=torch.float64) ** -skew
    cum = torch.cumsum(p / p.sum(), 0)
    e = torch.searchsorted(cum, _rand(g, n).double()).clamp_(max=of - 1)
    if of > 128:
        e = torch.randperm(of, generator=g, device=DEV)[e]            # the frequent ids of a vocabulary lie anywhere
    e = e.to(torch.int32)
    if drop:
        e[_rand(g, n) < drop / 100.0] = -1
    return e


def _rows(g, n, width, dtype):
    """Rows of very different magnitude, a few channels that stand out, and some rows of zeros (an atom without
    neighbours has a descriptor of zeros)."""
    x = _randn(g, n, width).mul_(torch.exp(_randn(g, n, 1)))
    x.mul_(torch.where(_rand(g, width) < 0.01, 8.0, 1.0))
    x[13::97] = 0.0
    return x.to(TYPES[dtype])


def _layers(g, experts, outer, inner):
    """Codes and scales of random weights: what a program keeps of a layer."""
    pairs = [_code(_randn(g, outer, inner) / math.sqrt(inner)) for _ in range(experts)]
    return torch.stack([c for c, _ in pairs]), torch.stack([s for _, s in pairs])


def prepare(case, seed):
    g, n, path = _gen(seed, 1), case["tokens"], case["path"]
    s = {"case": case}
    if path in ("gate", "gate_bwd"):
        s["logits"] = _logits(case, g)
        # as balancing moves it: small against the scores' range
        s["bias"] = 0.1 * _randn(g, case["experts"]) if case["bias"] else None
        if path == "gate_bwd":
            s["expert"] = _choose(s)[0]
            s["dweight"] = _randn(g, n, case["topk"])
    elif path in ("embed", "embed_bwd"):
        s["ids"] = _some(g, n, case["ids"], case["skew"], case["empty"])
        if path == "embed":
            s["table"] = _randn(g, case["ids"], case["width"]).to(TYPES[case["dtype"]])
        else:
            # of a mean over the batch, in the size that keeps 16-bit sums in range
            s["dy"] = (_rows(g, n, case["width"], "f32") / (8.0 * math.sqrt(n))).to(TYPES[case["dtype"]])
    else:
        s["x"] = _rows(g, n, case["inner"], case["dtype"])
        if path != "codes":
            s["codes"], s["scales"] = _layers(g, case.get("experts", 1), case["outer"], case["inner"])
            s["bias"] = _randn(g, case.get("experts", 1), case["outer"])
        if path == "expert":
            chosen = _some(g, n * case["topk"], case["experts"], case["skew"], case["drop"])
            s["offsets"], s["rows"], s["pos"] = _plan(chosen.view(n, -1), case["experts"])
    return s


def _plan(expert, experts):
    """Slots sorted by expert, ties by slot: offsets [E + 1], slot of each row, row of each slot (-1: dropped)."""
    e = expert.reshape(-1).long()
    kept = (e >= 0) & (e < experts)
    key, order = torch.sort(torch.where(kept, e, experts), stable=True)
    offsets = torch.searchsorted(key, torch.arange(experts + 1, device=DEV))
    at = torch.arange(len(e), device=DEV)
    pos = torch.empty_like(order)
    pos[order] = at
    return (offsets.to(torch.int32), torch.where(at < offsets[experts], order, -1).to(torch.int32),
            torch.where(kept, pos, -1).to(torch.int32).view(expert.shape))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2107_02103_amd as P
    case, path = s["case"], s["case"]["path"]
    if path in ("gate", "gate_bwd"):
        gate = P.Gate(case["experts"], case["topk"], score=case["score"], groups=case["groups"], keep=case["keep"],
                      best=case["best"], bias=s["bias"], renormalise=case["renorm"], scale=case["scale"])
        if path == "gate":
            expert, weight = gate(s["logits"])
            return {"expert": expert, "weight": weight}
        return {"dlogits": gate.backward(s["logits"], s["expert"], s["dweight"])}
    if path == "embed":
        return {"y": P.Embedding(s["table"], scale=case["scale"])(s["ids"])}
    if path == "embed_bwd":
        return {"dtable": P.Embedding.gradient(s["ids"], s["dy"], case["ids"], scale=case["scale"])}
    if path == "codes":
        return {"values": P.Mx4Rows.from_rows(s["x"]).values(TYPES[case["out"]])}
    layer = P.Mx4Linear(s["codes"], s["scales"], case["inner"], s["bias"])
    route = P.Route.from_plan(s["offsets"], s["rows"], s["pos"]) if path == "expert" else None
    return {"y": layer(s["x"], route=route, dtype=TYPES[case["out"]])}


def _scores(z, kind):
    """Softmax over the open experts, or sigmoids; 0 where an expert is closed."""
    if kind == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - torch.where(top == -INF, 0.0, top))
    total = p.sum(1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total)


def _choose(s):
    """Experts of each token and their weights: the values that decide are held in 64 bits, ties go to the lowest
    expert."""
    case, z = s["case"], s["logits"].double()
    n, E, G, k = case["tokens"], case["experts"], case["groups"], case["topk"]
    score = _scores(z, case["score"])
    c = score if s["bias"] is None else score + s["bias"].double()
    c = torch.where(z == -INF, -INF, c)
    if G > 1:
        best = torch.sort(c.view(n, G, E // G), dim=2, descending=True).values[:, :, :case["best"]]
        value = torch.where((best == -INF).all(2), -INF, torch.where(best == -INF, 0.0, best).sum(2))
        order = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :case["keep"]]
        kept = torch.zeros((n, G), dtype=torch.bool, device=DEV).scatter_(1, order, True)
        c = torch.where(kept[:, :, None], c.view(n, G, -1), -INF).view(n, E)
    value, expert = torch.sort(c, dim=1, descending=True, stable=True)
    live = value[:, :k] > -INF
    w = torch.where(live, score.gather(1, expert[:, :k]), 0.0)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total == 0, 1.0, total)
    return torch.where(live, expert[:, :k], -1).to(torch.int32), (w * case["scale"]).float()


def _gate_bwd(s):
    case, score = s["case"], _scores(s["logits"].float(), s["case"]["score"])
    live = s["expert"] >= 0
    at = s["expert"].clamp(min=0).long()
    mine = torch.where(live, score.gather(1, at), 0.0)
    d = torch.where(live, s["dweight"], 0.0) * case["scale"]
    if case["renorm"]:
        total = mine.sum(1, keepdim=True)
        one = torch.where(total == 0, 1.0, total)
        d = torch.where(live & (total > 0), (d - (d * mine).sum(1, keepdim=True) / one) / one, 0.0)
    ds = torch.zeros_like(score).scatter_add_(1, at, d)
    if case["score"] == "sigmoid":
        dz = ds * score * (1.0 - score)
    else:
        dz = score * (ds - (d * mine).sum(1, keepdim=True))
    return dz.to(s["logits"].dtype)


def _code(x):
    """Codes [rows, padded / 2] (two in a byte, the lower first) and scales [padded / 256, rows, 8] of rows."""
    n, K = x.shape
    ld = -(-K // STEP) * STEP
    v = torch.zeros((n, ld), device=DEV)
    v[:, :K] = x
    v = v.view(n, ld // BLOCK, BLOCK)
    a = v.abs().amax(2)
    e = ((a.view(torch.int32) + (1 << 21)) >> 23) - 2              # exponent of a, rounded up from 1.75 on, less two
    e = torch.where(a < TINY, 0, e)
    v = v * torch.where(a < TINY, 0.0, ((254 - e) << 23).view(torch.float32))[:, :, None]
    u = v.abs()
    q = (u > 0.25).to(torch.uint8)
    for bound, tie in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        q += (u >= bound) if tie else (u > bound)                  # ties to the even code
    q = (q + 8 * ((v < 0) & (q > 0)).to(torch.uint8)).view(n, ld)
    return q[:, 0::2] + 16 * q[:, 1::2], e.to(torch.uint8).view(n, ld // STEP, 8).transpose(0, 1).contiguous()


def _decode(codes, scales, K):
    """The values that codes and scales stand for, in 32 bits."""
    q = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1).long()
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    v = torch.cat([table, -table])[q]
    scale = torch.exp2(scales.transpose(0, 1).reshape(codes.shape[0], -1).float() - 127.0)
    return (v.view(v.shape[0], -1, BLOCK) * scale[:, :, None]).view(v.shape[0], -1)[:, :K]


def _run_plain(s):
    case, path = s["case"], s["case"]["path"]
    if path == "gate":
        expert, weight = _choose(s)
        return {"expert": expert, "weight": weight}
    if path == "gate_bwd":
        return {"dlogits": _gate_bwd(s)}
    if path == "embed":
        y = s["table"][s["ids"].clamp(min=0).long()].float() * case["scale"]
        return {"y": torch.where((s["ids"] >= 0)[:, None], y, 0.0).to(s["table"].dtype)}
    if path == "embed_bwd":
        ids, dy, f64 = s["ids"].long(), s["dy"], torch.float64
        if case["ids"] <= 64:
            d = torch.stack([torch.where((ids == v)[:, None], dy, 0.0).sum(0, dtype=f64) for v in range(case["ids"])])
        else:
            d = torch.zeros((case["ids"] + 1, case["width"]), dtype=f64, device=DEV)
            d = d.index_add_(0, torch.where(ids < 0, case["ids"], ids), dy.double())[:-1]
        return {"dtable": (d * case["scale"]).to(s["dy"].dtype)}
    out = TYPES[case["out"]]
    K = case["inner"]
    x = _decode(*_code(s["x"]), K)
    if path == "codes":
        return {"values": x.to(out)}
    if path == "linear":
        return {"y": (x @ _decode(s["codes"][0], s["scales"][0], K).t() + s["bias"][0]).to(out)}
    x = x[torch.div(s["rows"].clamp(min=0), case["topk"], rounding_mode="floor").long()]
    y = torch.zeros((len(x), case["outer"]), device=DEV)
    bounds = s["offsets"].tolist()
    for e, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):    # one product for each expert that has rows
        if hi > lo:
            y[lo:hi] = x[lo:hi] @ _decode(s["codes"][e], s["scales"][e], K).t() + s["bias"][e]
    return {"y": y.to(out)}


# ---------------------------------------------------------------------------
# the same values in 64 bits, from the definition
# ---------------------------------------------------------------------------
def _first_best(c):
    """The largest of each row and the lowest place that has it."""
    top = c.amax(1, keepdim=True)
    place = torch.where(c == top, torch.arange(c.shape[1], device=DEV), c.shape[1]).amin(1, keepdim=True)
    return top, place


def _exact_gate(s):
    """Experts one after the other, each the best that is left; scores from logarithms."""
    case, z = s["case"], s["logits"].double()
    n, E, G = case["tokens"], case["experts"], case["groups"]
    if case["score"] == "softmax":
        score = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)).nan_to_num(nan=0.0)
    else:
        score = torch.sigmoid(z)
    c = score + (0.0 if s["bias"] is None else s["bias"].double())
    c[z == -INF] = -INF
    if G > 1:
        value = torch.full((n, G), -INF, dtype=torch.float64, device=DEV)
        for g in range(G):
            left = c[:, g * (E // G):(g + 1) * (E // G)].clone()
            for _ in range(min(case["best"], E // G)):
                top, at = _first_best(left)
                live = (top > -INF)[:, 0]
                value[live, g] = value[live, g].nan_to_num(neginf=0.0, posinf=0.0) + top[live, 0]
                left.scatter_(1, at, -INF)
        out = torch.ones((n, G), dtype=torch.bool, device=DEV)
        for _ in range(case["keep"]):
            top, at = _first_best(value)
            out.scatter_(1, at, False)
            value.scatter_(1, at, -INF)
            value[top[:, 0] == -INF] = -INF
        c[out.repeat_interleave(E // G, 1)] = -INF
    expert = torch.full((n, case["topk"]), -1, dtype=torch.int32, device=DEV)
    w = torch.zeros((n, case["topk"]), dtype=torch.float64, device=DEV)
    for j in range(case["topk"]):
        top, at = _first_best(c)
        live = (top > -INF)[:, 0]
        expert[live, j] = at[live, 0].to(torch.int32)
        w[live, j] = score.gather(1, at)[live, 0]
        c.scatter_(1, at, -INF)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return expert, w * case["scale"]


def _exact_gate_bwd(s):
    """The derivative of sum(dweight * weight) by 64-bit differentiation of the weights at the given choices."""
    case = s["case"]
    z = s["logits"].double().requires_grad_()
    if case["score"] == "softmax":
        closed = z == -INF
        none = closed.all(1, keepdim=True)
        score = torch.softmax(torch.where(none, 0.0, z), 1)
    else:
        score = torch.sigmoid(z)
    live = s["expert"] >= 0
    w = torch.where(live, score.gather(1, s["expert"].clamp(min=0).long()), 0.0)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    (w * s["dweight"].double() * case["scale"]).sum().backward()
    return z.grad


def _exact_values(x):
    """What the codes of rows stand for: the block's power of two from its largest magnitude (as a 32-bit number),
    multiples of the step of each binade, ties to even."""
    n, K = x.shape
    pad = -K % BLOCK
    v = torch.nn.functional.pad(x.float().double(), (0, pad)).view(n, -1, BLOCK)
    a = v.abs().amax(2, keepdim=True)
    m, e = torch.frexp(a)
    scale = torch.exp2((e - 3 + (m >= 0.875)).double())
    u = v.abs() / scale
    step = torch.where(u < 2, 0.5, torch.where(u < 4, 1.0, 2.0))
    u = (torch.round(u / step) * step).clamp(max=6.0)
    return torch.where(a < TINY, 0.0, torch.sign(v) * u * scale).view(n, -1)[:, :K]


def _exact_weights(codes, scales, K):
    value = torch.tensor([(-1) ** (i >> 3) * [0, 1, 2, 3, 4, 6, 8, 12][i & 7] / 2 for i in range(16)], device=DEV,
                         dtype=torch.float64)
    rows = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=DEV)
    rows[:, 0::2] = value[(codes % 16).long()]
    rows[:, 1::2] = value[torch.div(codes, 16, rounding_mode="floor").long()]
    scale = 2.0 ** (scales.double() - 127.0)
    for step in range(scales.shape[0]):
        for b in range(8):
            at = step * STEP + b * BLOCK
            rows[:, at:at + BLOCK] *= scale[step, :, b:b + 1]
    return rows[:, :K]


def _exact_layer(s, tokens, expert):
    case = s["case"]
    w = _exact_weights(s["codes"][expert], s["scales"][expert], case["inner"]).t().contiguous()
    y = torch.empty((len(tokens), case["outer"]), dtype=torch.float64, device=DEV)
    for i in range(0, len(tokens), 65536):
        y[i:i + 65536] = _exact_values(s["x"][tokens[i:i + 65536]]) @ w + s["bias"][expert].double()
    return y


def exact(case, seed):
    s, path, n = prepare(case, seed), case["path"], case["tokens"]
    if path == "gate":
        expert, weight = _exact_gate(s)
        return {"expert": expert, "weight": weight}
    if path == "gate_bwd":
        return {"dlogits": _exact_gate_bwd(s)}
    if path == "embed":
        y = torch.zeros((n, case["width"]), dtype=torch.float64, device=DEV)
        y[s["ids"] >= 0] = case["scale"] * s["table"].double()[s["ids"][s["ids"] >= 0].long()]
        return {"y": y}
    if path == "embed_bwd":
        # tokens in the order of their ids; the sum of an id's run is the difference of two running sums
        ids, order = torch.sort(s["ids"], stable=True)
        bounds = torch.searchsorted(ids, torch.arange(case["ids"] + 1, device=DEV, dtype=torch.int32))
        d = torch.empty((case["ids"], case["width"]), dtype=torch.float64, device=DEV)
        wide = max(1, (1 << 28) // max(n, case["ids"]))
        for c in range(0, case["width"], wide):
            run_sum = torch.cumsum(s["dy"][:, c:c + wide][order].double(), 0)
            run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
            d[:, c:c + wide] = case["scale"] * (run_sum[bounds[1:]] - run_sum[bounds[:-1]])
        return {"dtable": d}
    if path == "codes":
        y = torch.empty((n, case["inner"]), dtype=torch.float64, device=DEV)
        for i in range(0, n, 65536):
            y[i:i + 65536] = _exact_values(s["x"][i:i + 65536])
        return {"values": y}
    if path == "linear":
        return {"y": _exact_layer(s, torch.arange(n, device=DEV), 0)}
    k = case["topk"]
    y = torch.zeros((n * k, case["outer"]), dtype=torch.float64, device=DEV)
    off = s["offsets"].tolist()
    for e in range(case["experts"]):
        if off[e + 1] > off[e]:
            y[off[e]:off[e + 1]] = _exact_layer(s, s["rows"][off[e]:off[e + 1]].long() // k, e)
    return {"y": y}
