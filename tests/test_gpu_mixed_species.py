"""The fitting nets of several species behind a routing (examples/mixed_species.py)
against the oracle's net of each species.

float64: 1e-12 of an atom's largest value, as for one net.  8 bits: a product of
codes is off by s / sqrt(12) per element of either side, about 0.8% of the row's
root mean square each (rows of 64 to 1,600 values reach 3 to 3.5 times theirs),
1.1% together; three products forward and three back add up to sqrt(6) times
that, 2.8%.  The bounds are four times as wide."""
import importlib.util
import os

import numpy as np
import pytest

import oracle.experts as ox
import oracle.fitting as fn
from oracle import cref
from oracle.table import build_tables
from synth import make_inputs
from synth.configs import get_config
from synth.system import random_fitting_net

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ms():
    spec = importlib.util.spec_from_file_location("mixed_species", os.path.join(ROOT, "examples", "mixed_species.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _oracle(D, nets, species, weight):
    n, k = species.shape
    E, dD, dw = np.zeros(n), np.zeros_like(D), np.zeros((n, k))
    for a, net in enumerate(nets):
        e, g = fn.forward(D, net)[0], fn.backward(D, net)
        for j in range(k):
            mine = species[:, j] == a
            w = np.ones(n) if weight is None else weight[:, j]
            E += np.where(mine, w * e, 0.0)
            dD += np.where(mine, w, 0.0)[:, None, None] * g
            dw[:, j] += np.where(mine, e, 0.0)
    return E, dD, dw


@pytest.mark.parametrize("n,m1,m2,width,k,nspec", [(300, 100, 16, 240, 1, 3), (77, 16, 4, 240, 2, 3), (5, 100, 16, 240, 2, 4),
                                                   (1, 16, 4, 240, 1, 2), (60, 7, 3, 33, 2, 2)])
def test_mixed_fitting(ms, n, m1, m2, width, k, nspec):
    rng = np.random.default_rng(n)
    nets = [random_fitting_net(rng, m1 * m2, (width,) * 3) for _ in range(nspec)]
    species = rng.integers(0, nspec, (n, k)).astype(np.int32)
    if k > 1:
        species[rng.random(n) < 0.3, 1] = -1
    weight = rng.random((n, k)) if k > 1 else None
    D = rng.standard_normal((n, m1, m2))
    want = _oracle(D, nets, species, weight)
    fit = ms.MixedFitting(nets, "f64")
    sp = torch.from_numpy(species).cuda()
    w = None if weight is None else torch.from_numpy(weight).cuda()
    E, dD, dw = fit(torch.from_numpy(D).cuda(), sp, w)
    fit.close()
    assert np.abs(E.cpu().numpy() - want[0]).max() <= 1e-12 * np.abs(want[0]).max()
    g = np.abs(want[1]).reshape(n, -1).max(1)
    assert (np.abs(dD.cpu().numpy() - want[1]).reshape(n, -1).max(1) <= 1e-12 * g).all()
    if k > 1:
        assert np.abs(dw.cpu().numpy() - want[2]).max() <= 1e-12 * np.abs(want[2]).max()
    for dt in (torch.float32, torch.float64):
        fit = ms.MixedFitting(nets, "int8")
        w = None if weight is None else torch.from_numpy(weight).to(dt).cuda()
        if dt == torch.float64 and w is not None:
            continue                                        # the 8-bit nets' rows are float32
        E, dD, dw = fit(torch.from_numpy(D).to(dt).cuda(), sp, w)
        spread = np.sqrt(np.mean((want[0] - want[0].mean()) ** 2)) if n > 10 else 1.0
        assert np.sqrt(np.mean((E.cpu().numpy() - want[0]) ** 2)) <= 0.11 * spread
        assert np.linalg.norm(dD.double().cpu().numpy() - want[1]) <= 0.11 * np.linalg.norm(want[1])
        if k > 1:
            assert np.linalg.norm(dw.cpu().numpy() - want[2]) <= 0.11 * np.linalg.norm(want[2])


def _by_codes(D, nets, species):
    """The 8-bit nets in 64 bits around the same codes: energies and dE/dD."""
    x = D.reshape(len(D), -1).astype(np.float64)
    E, dD = np.zeros(len(x)), np.zeros_like(x)

    def product(rows, W):
        qx, sx = ox.codes(rows)
        qw, sw = ox.codes(W.T)
        return ox.product(qx, sx, qw[None], sw[None])[0]

    for a, net in enumerate(nets):
        mine = species == a
        W, b = net["W"], [v.astype(np.float32).astype(np.float64) for v in net["b"]]
        t = [np.tanh(product(x[mine], W[0]) + b[0])]
        h = t[0]
        for l in (1, 2):
            t.append(np.tanh(product(h, W[l]) + b[l]))
            h = h + t[l]
        E[mine] = h @ net["w_out"] + net["b_out"]
        g = np.broadcast_to(net["w_out"], h.shape)
        for l in (2, 1):
            g = g + product((1 - t[l] ** 2) * g, W[l].T)
        dD[mine] = product((1 - t[0] ** 2) * g, W[0].T)
    return E, dD.reshape(D.shape)


def _tiny_alloy():
    """The system, its descriptors, and nets whose first layer expects descriptors of that size."""
    x = make_inputs(get_config("tiny_alloy"), with_grad=False)
    _, D = cref.Problem(x.em, x.nlist, x.atype, build_tables(x), x.cfg.sel, x.cfg.m2).forward()
    rng = np.random.default_rng(2)
    nets = [random_fitting_net(rng, x.cfg.m1 * x.cfg.m2) for _ in range(x.cfg.ntypes)]
    for net in nets:
        net["W"][0] /= np.sqrt(np.mean(D ** 2))
    return x, D, nets


def test_8_bit_nets_against_their_codes(ms):
    # float32's tanh is off by 2^-22 and moves a code by one (of 127) in 6e-5 of the elements, so in 7% of the rows of
    # five products; one code is 1.7e-3 of a row of 240: sqrt(0.07) * 1.7e-3 of the norm, four times that allowed
    x, D, nets = _tiny_alloy()
    D = D.astype(np.float32)
    fit = ms.MixedFitting(nets, "int8")
    E, dD, _ = fit(torch.from_numpy(D).cuda(), torch.from_numpy(x.atype).cuda())
    Er, dr = _by_codes(D, nets, x.atype)
    assert np.linalg.norm(E.cpu().numpy() - Er) <= 2e-3 * np.linalg.norm(Er)
    assert np.linalg.norm(dD.cpu().numpy() - dr) <= 2e-3 * np.linalg.norm(dr)


def test_positions_to_forces(ms):
    x, _, nets = _tiny_alloy()
    got = {}
    # one net for all species: the routed nets are that one net
    for name, ns, species in (("one", nets[:1], np.zeros(len(x.atype))), ("same", nets[:1] * 3, x.atype),
                              ("own", nets, x.atype)):
        fit = ms.MixedFitting(ns, "f64")
        got[name] = ms.energies_and_forces(x, fit, torch.from_numpy(species.astype(np.int32)).cuda())
        fit.close()
    for a, b in zip(got["one"][:2], got["same"][:2]):
        assert float((a - b).abs().max()) <= 1e-12 * float(a.abs().max())
    fit = ms.MixedFitting(nets, "int8")
    E8, F8, _ = ms.energies_and_forces(x, fit, torch.from_numpy(x.atype).cuda())
    E, F, _ = got["own"]
    assert float((F8 - F).norm()) <= 0.11 * float(F.norm())
    assert float((E8.double() - E).norm()) <= 0.11 * float((E - E.mean()).norm())
