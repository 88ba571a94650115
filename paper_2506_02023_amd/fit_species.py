"""Fits a scale and a shift of the atoms' energies for each species to reference energies of structures.

    python -m paper_2506_02023_amd.fit_species [--structures 64] [--cells 5] [--steps 400] [--lr 0.05] [--max-norm 1.0] [--seed 0]

Adapting a potential to energies of another reference method begins with this: the potential stays as it is, and
E_pred = sum over a structure's atoms of scale[z_i] e_i + shift[z_i] is fitted to the structures' energies.  The atoms'
energies e_i come from mlip_build_graph and mlip_forward, once; every step of the fit then looks the species' rows up
(mlip_embed), sums atoms by structure and gradients by species (mlip_embed_grad), bounds the gradient's norm (mlip_clip_grads) and makes
an Adam update in torch arithmetic.  Structures of all sizes lie one after another in one batch.  The reference energies
here are synthetic: the model's own with hidden scales and shifts.  The fit is judged by the error of the structures' energies that is left; scale and
shift of a species by themselves are found only as far as its atoms' energies differ, which here is little.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def loss_and_gradient(table, atom_e, species, structure, atoms_of, e_ref):
    """(error per atom of every structure [B], gradient of half their mean square with respect to the table [S, 2]).

    table: [S, 2], scale and shift of each species; atom_e [n]; species, structure: int32 [n]; atoms_of, e_ref: [B]."""
    import torch

    import paper_2506_02023_amd as M

    rows = M.mlip_embed(table, species)
    energy = M.mlip_embed_grad(torch.addcmul(rows[:, 1], rows[:, 0], atom_e), structure, len(e_ref))
    error = (energy - e_ref) / atoms_of
    atom_bar = M.mlip_embed(error / atoms_of, structure, 1.0 / len(e_ref))
    return error, M.mlip_embed_grad(torch.stack([atom_bar * atom_e, atom_bar], 1), species, table.shape[0])


def fit(table, atom_e, species, structure, atoms_of, e_ref, steps, lr, max_norm):
    """`steps` Adam steps on the table, in place; returns the root-mean-square error per atom before each.

    A species' energies lie close together, so its scale and shift do almost the same to a structure's energy.  The steps are made in the scale times the
    energies' standard deviation and the shift at their mean, which are told apart at once."""
    import torch

    import paper_2506_02023_amd as M

    S = table.shape[0]
    counts = M.mlip_embed_grad(torch.ones(1, device="cuda").expand(len(species)), species, S).clamp(min=1.0)
    mean = M.mlip_embed_grad(atom_e, species, S) / counts
    centred = atom_e - M.mlip_embed(mean, species)
    spread = (M.mlip_embed_grad(centred.square(), species, S) / counts).sqrt()
    spread = torch.where(spread > 1e-6, spread, 1.0)
    centred /= M.mlip_embed(spread, species)
    inner = torch.stack([table[:, 0] * spread, table[:, 1] + table[:, 0] * mean], 1)

    first, second = torch.zeros_like(inner), torch.zeros_like(inner)
    errors = []
    for k in range(1, steps + 1):
        error, grad = loss_and_gradient(inner, centred, species, structure, atoms_of, e_ref)
        M.mlip_clip_grads([grad], max_norm)
        first.lerp_(grad, 0.1)
        second.lerp_(grad * grad, 0.01)
        rate = lr * min(1.0, 4.0 * (1.0 - k / (steps + 1)))      # the last quarter runs down
        inner -= rate * (first / (1 - 0.9 ** k)) / ((second / (1 - 0.99 ** k)).sqrt() + 1e-12)
        errors.append(error.square().mean().sqrt())              # read back after the loop: no host synchronisation inside a step
    table[:, 0] = inner[:, 0] / spread
    table[:, 1] = inner[:, 1] - table[:, 0] * mean
    return [float(e) for e in errors]


def structures_of(count, cells, n_species, seed):
    """(positions, cell, species) of jittered fcc structures of different compositions, the last with fewer cells than the first."""
    import numpy as np

    import workloads as wl

    rng = np.random.default_rng(seed)
    out = []
    for k in range(count):
        positions, cell, _ = wl.fcc_lattice(max(3, cells - k * 2 // count), 0.1, n_species, seed * 1000 + k)
        out.append((positions, cell, rng.choice(n_species, len(positions), p=rng.dirichlet(np.ones(n_species))).astype(np.int32)))
    return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--structures", type=int, default=64)
    ap.add_argument("--cells", type=int, default=5, help="fcc cells per side of the largest structures")
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--lr", type=float, default=0.05)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()

    import numpy as np
    import torch

    import paper_2506_02023_amd as M
    import workloads as wl

    c = wl.make_config(1, n=3)
    weights, S = M.Weights(c["weights"], c["p"]), c["S"]
    atom_e, species, g = [], [], None
    for positions, cell, z in structures_of(args.structures, args.cells, S, args.seed):
        spec = torch.as_tensor(z, device="cuda")
        g = M.mlip_build_graph(torch.as_tensor(positions, device="cuda"), cell, spec, c["r_cut"], graph=g)
        atom_e.append(M.mlip_forward(g, weights)[2])
        species.append(spec)
    sizes = torch.tensor([len(s) for s in species], device="cuda")
    structure = torch.repeat_interleave(torch.arange(len(species), device="cuda", dtype=torch.int32), sizes)
    atom_e, species, atoms_of = torch.cat(atom_e), torch.cat(species), sizes.float()

    rng = np.random.default_rng(args.seed)
    hidden = np.stack([rng.uniform(0.7, 1.3, S), rng.uniform(-3.0, 3.0, S)], 1)
    hidden = torch.as_tensor(hidden, dtype=torch.float32, device="cuda")
    rows = M.mlip_embed(hidden, species)
    e_ref = M.mlip_embed_grad(rows[:, 0] * atom_e + rows[:, 1], structure, len(sizes))

    table = torch.tensor([[1.0, 0.0]], device="cuda").repeat(S, 1)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    errors = fit(table, atom_e, species, structure, atoms_of, e_ref, args.steps, args.lr, args.max_norm)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / max(args.steps, 1) * 1e3
    print(f"{len(sizes)} structures, {len(species)} atoms, {S} species: {args.steps} steps of {ms:.3f} ms")
    if errors:
        print(f"error per atom {errors[0]:.3e} -> {errors[-1]:.3e}")
    print(f"largest error of the {2 * S} parameters {float((table - hidden).abs().max()):.2e}")


if __name__ == "__main__":
    main()
