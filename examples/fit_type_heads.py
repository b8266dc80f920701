"""Fits energy heads with weights of each element type to a model's energies.

    python examples/fit_type_heads.py [--steps 200] [--hidden 64] [--frames 4]

The frames are a five-element alloy at random displacements; the model's
descriptors of their atoms go through three layers whose weights belong to the
atom's element (two with SiLU, the second with a residual; the third gives the
energy), and the model's own energies of the atoms, of all types alike, are what
the heads learn.  The rows are grouped once, since a frame's species do not
change; the matrices are updated by Muon and the rest by Adam.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_19041_amd as dp  # noqa: E402
import synth  # noqa: E402


def frames(count, device, model_name="small", reps=6):
    """Descriptors [n, D], energies [n] and element types [n] of the atoms of all frames."""
    spec, weights = synth.model_weights(model_name)
    model = dp.Model(synth.pack_blob(spec, weights))
    rows = []
    for seed in range(count):
        s = synth.bcc_hea(reps=reps, jitter=0.04 + 0.03 * seed, seed=seed)
        pos = torch.tensor(s.pos, dtype=torch.float64, device=device)
        species = torch.tensor(s.species, dtype=torch.int32, device=device)
        pairs = dp.build_neighbors(pos, s.cell, s.pbc, spec.r_c + 1.0)
        energy, _, _ = model.compute_energy_forces(pos, species, s.cell, s.pbc, spec.r_c, *pairs)
        rows.append((model.debug_stages(s.n)[1], energy.float(), species))
    x, energy, species = (torch.cat(parts) for parts in zip(*rows))
    return x / x.square().mean(0).sqrt().clamp(min=1e-6), energy, species   # calibrated to order one


class Heads:
    """Three layers with weights of each of ``types`` element types."""

    def __init__(self, width, hidden, types, species, seed=0):
        g = torch.Generator(device=species.device).manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device=species.device) * shape[1] ** -0.5

        self.ptr, self.order = dp.group_rows(species, types)
        self.w = [normal(types, width, hidden), normal(types, hidden, hidden), normal(types, hidden, 1)]
        self.b = [torch.zeros(types, w.shape[2], device=species.device) for w in self.w]

    def _layer(self, i, x, **how):
        return dp.grouped_linear(x, self.w[i], self.ptr, self.order, bias=self.b[i], **how)

    def energies(self, x):
        """Energies of the rows, and what ``gradients`` needs."""
        y1, z1 = self._layer(0, x, activation="silu", preact=True)
        y2, z2 = self._layer(1, y1, activation="silu", residual=True, preact=True)
        return self._layer(2, y2)[:, 0], (x, y1, z1, y2, z2)

    def gradients(self, de, kept):
        """(dw, db) of every layer from the gradient of the rows' energies."""
        x, y1, z1, y2, z2 = kept

        def back(i, dy, x, **how):
            return dp.grouped_linear_backward(dy, x, self.w[i], self.ptr, self.order, **how)

        d2, dw2, db2 = back(2, de[:, None], y2)
        d1, dw1, db1 = back(1, d2, y1, preact=z2, residual=True)
        _, dw0, db0 = back(0, d1, x, preact=z1, need=(False, True, True))
        return [dw0, dw1, dw2], [db0, db1, db2]


def fit(x, target, species, types, hidden=64, steps=200, lr=0.02):
    """The heads, and the root mean square error in eV after each tenth of the steps."""
    heads = Heads(x.shape[1], hidden, types, species)
    matrices, rest = heads.w[:2], heads.w[2:] + heads.b
    momenta = [torch.zeros_like(w) for w in matrices]
    adam = torch.optim.Adam(rest, lr=1e-2)
    errors = []
    for step in range(steps + 1):
        rate = 1.0 - step / (steps + 1)
        e, kept = heads.energies(x)
        off = e - target
        if step % max(1, steps // 10) == 0:
            errors.append(off.square().mean().sqrt().item())
        dw, db = heads.gradients(off * (2.0 / len(off)), kept)
        dp.muon_step(matrices, dw[:2], momenta, lr=lr * rate)
        for p, g in zip(rest, dw[2:] + db):
            p.grad = g
        for group in adam.param_groups:
            group["lr"] = 1e-2 * rate
        adam.step()
    return heads, errors


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--hidden", type=int, default=64)
    ap.add_argument("--frames", type=int, default=4)
    a = ap.parse_args()
    x, energy, species = frames(a.frames, torch.device("cuda", 0))
    target = energy - energy.mean()
    print(f"{len(x)} atoms of {len(species.unique())} elements, {x.shape[1]} descriptors, "
          f"energies off their mean by {target.square().mean().sqrt().item():.4f} eV")
    _, errors = fit(x, target, species, 118, a.hidden, a.steps)
    for i, err in enumerate(errors):
        print(f"step {i * max(1, a.steps // 10):5d}  rms error {err:.5f} eV", flush=True)


if __name__ == "__main__":
    main()
