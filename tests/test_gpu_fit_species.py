"""The fit of per-species scales and shifts: its gradient against autograd in 64 bits, and what a fit recovers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _batch(seed, n=3000, B=17, S=5):
    import torch
    rng = np.random.default_rng(seed)
    structure = np.sort(rng.integers(0, B, n))
    mix = rng.dirichlet(np.ones(S), B)
    species = np.array([rng.choice(S, p=mix[b]) for b in structure])
    dev = dict(device="cuda")
    atom_e = torch.as_tensor(rng.normal(-2.0, 0.5, n), dtype=torch.float32, **dev)
    atoms_of = torch.as_tensor(np.bincount(structure, minlength=B), dtype=torch.float32, **dev)
    e_ref = torch.as_tensor(rng.normal(-2.0, 1.0, B), dtype=torch.float32, **dev) * atoms_of
    table = torch.as_tensor(rng.normal(1.0, 0.3, (S, 2)), dtype=torch.float32, **dev)
    return (table, atom_e, torch.as_tensor(species, dtype=torch.int32, **dev), torch.as_tensor(structure, dtype=torch.int32, **dev),
            atoms_of, e_ref)


def test_gradient_against_autograd():
    """Every quantity is a sum of at most 3000 products; with u = 2^-24 an energy is off by at most 1030 u of the sum of its terms' magnitudes (which a
    structure's error inherits), a gradient by that and as much again: 5000 u of the magnitudes bounds both."""
    import torch
    from paper_2506_02023_amd import fit_species as fs
    table, atom_e, species, structure, atoms_of, e_ref = _batch(1)
    error, grad = fs.loss_and_gradient(table, atom_e, species, structure, atoms_of, e_ref)
    t = table.double().cpu().requires_grad_()
    e, z, b, n, ref = (x.cpu() for x in (atom_e.double(), species.long(), structure.long(), atoms_of.double(), e_ref.double()))
    terms = t[z, 0] * e + t[z, 1]
    err = (torch.zeros_like(ref).index_add(0, b, terms) - ref) / n
    (0.5 * err.square().mean()).backward()
    off = 5000 * 2.0 ** -24
    size = (torch.zeros_like(ref).index_add(0, b, (t[z, 0] * e).abs() + t[z, 1].abs()) + ref.abs()) / n     # per atom
    assert (error.cpu().double() - err).abs().le(off * size).all()
    weight = (size / n / len(n))[b]
    most = torch.zeros_like(t).index_add(0, z, torch.stack([weight * e.abs(), weight], 1))
    assert (grad.cpu().double() - t.grad).abs().le(off * most).all()


def test_fit_recovers_hidden_parameters():
    """Reference energies made with other scales and shifts: the fit's error falls below a hundredth of where it began."""
    import torch
    import paper_2506_02023_amd as M
    from paper_2506_02023_amd import fit_species as fs
    table, atom_e, species, structure, atoms_of, _ = _batch(2, B=60)
    rows = M.mlip_embed(table, species)
    e_ref = M.mlip_embed_grad(rows[:, 0] * atom_e + rows[:, 1], structure, len(atoms_of))
    start = torch.tensor([[1.0, 0.0]], device="cuda").repeat(len(table), 1)
    errors = fs.fit(start, atom_e, species, structure, atoms_of, e_ref, 400, 0.05, 1.0)
    assert errors[-1] < 0.01 * errors[0]
