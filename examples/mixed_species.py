"""One fitting net for each species, in float64 or in 8-bit integers, with mixed atoms.

    python examples/mixed_species.py [--config alcumg32000] [--mixed 0.1]

The descriptors of all atoms are routed to the net of their species and their
energies and gradients brought back.  An atom may also be a mixture of species,
E_i = sum_j w_ij E^(a_ij)(D_i), as on the way from one species to another in
free-energy calculations; dE/dw_ij is what such a calculation integrates.

float64: rows sorted by species, each species' rows through
dpc_fitting_fwd_bwd.  8 bits: every layer one call for all species, forward
and for the gradient, whose errors (about 1% of a product) suit searches and
members of an ensemble rather than dynamics: forces within 1 to 2% of their norm
where the nets expect descriptors of the size they have (as trained ones do, and
as the first layer is divided here).  Behind saturated layers they are wrong: with
random nets on the descriptors as they come the error is as large as the forces."""
import argparse
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2107_02103_amd as P  # noqa: E402


class MixedFitting:
    """Fitting nets {"W", "b", "w_out", "b_out"} of all species (three layers of
    one width, the form of dpc_fitting_net)."""

    def __init__(self, nets, precision="f64", device="cuda"):
        if precision not in ("f64", "int8"):
            raise ValueError("precision is f64 or int8")
        self.nspecies, self.precision = len(nets), precision
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
        self.width = nets[0]["w_out"].shape[0]
        self.w_out = dev(np.stack([n["w_out"] for n in nets]))
        self.b_out = dev(np.array([n["b_out"] for n in nets]))
        W = [dev(np.stack([n["W"][l] for n in nets])) for l in range(3)]
        b = [dev(np.stack([n["b"][l] for n in nets])) for l in range(3)]
        if precision == "int8":
            # codes of W^T (rows are output channels) and, for the gradient, of W
            self.layers = [P.Int8Linear.from_weight(w.transpose(1, 2), c) for w, c in zip(W, b)]
            self.back = [P.Int8Linear.from_weight(w) for w in W]
            self.w_out, self.b_out = self.w_out.float(), self.b_out.float()
            return
        self.W, self.b, self.blas, self.nets = W, b, P.RocblasHandle(), []
        for a in range(self.nspecies):
            c = P.dpc_fitting_net()
            c.n_in, c.width, c.b_out = W[0].shape[1], self.width, nets[a]["b_out"]
            for l in range(3):
                c.W[l], c.b[l] = W[l][a].data_ptr(), b[l][a].data_ptr()
            c.w_out = self.w_out[a].data_ptr()
            self.nets.append(c)

    def __call__(self, D, species, weight=None):
        """Energies [n], dE/dD (shape of D) and dE/dweight [n, k] (None without
        weights) for descriptors D [n, M, M'] and species int32 [n] or [n, k]."""
        x = D.reshape(D.shape[0], -1)
        route = P.Route(species, self.nspecies)
        E, dx = self._rows8(x, route, species) if self.precision == "int8" else self._rows64(x, route)
        E = E[:, None]
        energy = route.combine(E, weight)
        dD = route.combine(dx, weight).view(D.shape)
        dw = None
        if weight is not None:
            _, dw = route.combine_backward(E, torch.ones_like(energy), weight, need_rows=False)
        return energy[:, 0], dD, dw

    def _rows64(self, x, route):
        rows = route.gather(x)
        E, dx = torch.zeros(len(rows), dtype=torch.float64, device=x.device), torch.zeros_like(rows)
        off = route.offsets.tolist()
        nb = P.dpc_fitting_workspace_bytes(max(hi - lo for lo, hi in zip(off, off[1:])), self.width)
        ws = torch.empty(nb, dtype=torch.uint8, device=x.device)
        for net, lo, hi in zip(self.nets, off, off[1:]):
            if hi > lo:
                P.dpc_fitting_fwd_bwd(torch.cuda.current_stream(), self.blas.value, hi - lo, net, rows[lo:hi], ws, nb,
                                      E[lo:hi], dx[lo:hi])
        return E, dx

    def _rows8(self, x, route, species):
        f32, off = torch.float32, route.offsets
        t = [torch.tanh(self.layers[0](x, route=route, dtype=f32))]
        h = t[0]
        for l in (1, 2):
            t.append(torch.tanh(self.layers[l](h, offsets=off)))
            h = h + t[l]
        # the last product and its gradient are one column: not worth 8 bits
        a = species.reshape(-1)[route.rows.clamp(min=0).long()].clamp(0, self.nspecies - 1).long()
        w_out = self.w_out[a]
        E = (h * w_out).sum(1) + self.b_out[a]
        g = w_out
        for l in (2, 1):
            g = g + self.back[l]((1 - t[l] * t[l]) * g, offsets=off)
        dx = self.back[0]((1 - t[0] * t[0]) * g, offsets=off)
        return E, dx

    def close(self):
        if self.precision == "f64":
            self.blas.close()


def descriptor_scale(x):
    """Root mean square of the system's descriptors."""
    op = P.SeATab(x.nets, x.lo, x.L1, x.L2, x.cfg.d1, x.cfg.d2, x.cfg.sel, x.cfg.m2)
    _, D = op.forward(*(torch.from_numpy(a).cuda() for a in (x.em, x.nlist, x.atype)))
    return float(D.square().mean().sqrt())


def energies_and_forces(x, fitting, species=None, weight=None):
    """Energies, forces and dE/dweight of a synthetic system (synth.make_inputs): descriptor, routed fitting nets,
    backward to forces; in float64, or in float32 around the 8-bit nets."""
    c = x.cfg
    wide = fitting.precision == "f64"
    mode, dt = (P.DPC_F64, torch.float64) if wide else (P.DPC_F32, torch.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    nlist, atype, coord, n = dev(x.nlist), dev(x.atype), dev(x.coords), len(x.atype)
    stats = [np.asarray(x.stats[k], np.float64) for k in ("mean", "sigma", "sigma_all")]
    s = torch.cuda.current_stream()
    op = P.SeATab(x.nets, x.lo, x.L1, x.L2, c.d1, c.d2, c.sel, c.m2, dtype=mode)
    em = torch.empty((n, c.nnei, 4), dtype=dt, device="cuda")
    P.dpc_env_mat_a(s, mode, n, c.ntypes, c.nnei, c.box, c.rc, c.rcs, *stats, coord, atype, nlist, em)
    T, D = op.forward(em, nlist, atype)
    energy, dD, dw = fitting(D, atype if species is None else species, weight)
    dR = op.backward(em, nlist, atype, op.descriptor_backward(T, dD))
    rev = torch.empty_like(nlist)
    P.dpc_nlist_reverse(s, n, c.ntypes, c.sel, c.box, coord, atype, nlist, rev)
    force = torch.empty((n, 3), dtype=torch.float64, device="cuda")
    P.dpc_force_a(s, mode, n, c.ntypes, c.nnei, c.box, c.rc, c.rcs, *stats[1:], coord, atype, nlist, rev, dR, force)
    return energy, force, dw


def main():
    from synth import make_inputs
    from synth.configs import get_config
    from synth.system import random_fitting_net
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="tiny_alloy")
    ap.add_argument("--mixed", type=float, default=0.1, help="share of atoms that are mixtures of two species")
    args = ap.parse_args()
    x = make_inputs(get_config(args.config), with_grad=False)
    c, rng = x.cfg, np.random.default_rng(0)
    nets = [random_fitting_net(rng, c.m1 * c.m2) for _ in range(c.ntypes)]
    scale = descriptor_scale(x)
    for net in nets:
        net["W"][0] /= scale                 # a trained net expects descriptors of the size they have
    # second choice: none (-1), or another species with weight 0.3
    other = np.where(rng.random(len(x.atype)) < args.mixed, (x.atype + 1) % c.ntypes, -1)
    other[other == x.atype] = -1
    species = torch.from_numpy(np.stack([x.atype, other], 1).astype(np.int32)).cuda()
    lam = torch.where(species[:, 1] >= 0, 0.3, 0.0)
    weight = torch.stack([1 - lam, lam], 1)
    out = {}
    for precision in ("f64", "int8"):
        fit = MixedFitting(nets, precision)
        out[precision] = energies_and_forces(x, fit, species, weight.to(torch.float64 if precision == "f64" else torch.float32))
        fit.close()
    (E, F, dw), (E8, F8, dw8) = out["f64"], out["int8"]
    print(f"{c.name}: {len(x.atype)} atoms, {int((species[:, 1] >= 0).sum())} of them mixtures of two of {c.ntypes} species")
    for name, a, b in (("energy", E, E8), ("force", F, F8), ("dE/dweight", dw, dw8)):
        a, b = a.double(), b.double()
        print(f"  {name}: 8-bit against float64, error {float((a - b).norm() / a.norm()):.2e} of the norm")


if __name__ == "__main__":
    main()
