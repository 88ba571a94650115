"""Lookup and gradient inside a torch autograd graph, against autograd's own index operations in 64 bits.

Tables, gradients and scales are small whole numbers and powers of two, so all values here are exact and compared for equality."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SIZES = [(40, 4, 5), (3000, 7, 33), (3000, 900, 12), (300, 3, 1)]


def _inputs(n, rows, width, dtype, id_dtype):
    import torch
    rng = np.random.default_rng([n, rows, width])
    table = torch.as_tensor(rng.integers(-4, 5, (rows, width)), dtype=dtype, device="cuda")
    ids = rng.integers(0, rows, n)
    ids[rng.random(n) < 0.2] = -1
    w = torch.as_tensor(rng.integers(-4, 5, (n, width)), dtype=dtype, device="cuda")
    return table, torch.as_tensor(ids, dtype=id_dtype, device="cuda"), w


def _reference(table, ids, scale):
    """The lookup in fp64 by torch"""
    import torch
    return torch.where((ids >= 0)[:, None], table[ids.long().clamp(min=0)] * scale, 0.0)


@pytest.mark.parametrize("n,rows,width", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("id_dtype", ["int32", "int64"])
def test_lookup_passes_the_gradient_on(n, rows, width, dtype, id_dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    table, ids, w = _inputs(n, rows, width, dt, getattr(torch, id_dtype))
    leaf = table.clone().requires_grad_()
    out = M.mlip_embed(leaf, ids, 0.5)
    assert out.requires_grad and torch.equal(out.detach(), M.mlip_embed(table, ids, 0.5))
    out.backward(w)
    ref = table.double().requires_grad_()
    _reference(ref, ids, 0.5).backward(w.double())
    assert leaf.grad.dtype == dt and torch.equal(leaf.grad, ref.grad.to(dt))


@pytest.mark.parametrize("n,rows,width", SIZES)
def test_sums_pass_the_gradient_on(n, rows, width):
    import torch
    import paper_2506_02023_amd as M
    _, ids, g = _inputs(n, rows, width, torch.float32, torch.int32)
    ids = torch.where(torch.arange(n, device="cuda", dtype=torch.int32) % 7 == 3, rows + 2, ids)     # ids without a row on both sides
    bar = torch.as_tensor(np.random.default_rng(n).integers(-4, 5, (rows, width)), dtype=torch.float32, device="cuda")
    leaf = g.clone().requires_grad_()
    out = M.mlip_embed_grad(leaf, ids, rows, 2.0)
    assert out.requires_grad and torch.equal(out.detach(), M.mlip_embed_grad(g, ids, rows, 2.0))
    out.backward(bar)
    there = (ids >= 0) & (ids < rows)
    assert torch.equal(leaf.grad, torch.where(there[:, None], bar[ids.long().clamp(0, rows - 1)] * 2.0, 0.0))


def test_vectors_and_second_derivatives():
    """The energy of a structure by a table's squares: its second derivative with respect to the table"""
    import torch
    import paper_2506_02023_amd as M
    ids = torch.tensor([0, 2, 2, -1, 1, 2], device="cuda")
    t = torch.tensor([1.0, -2.0, 3.0, 5.0], device="cuda", requires_grad=True)
    energy = M.mlip_embed(t, ids).square().sum()
    first, = torch.autograd.grad(energy, t, create_graph=True)
    assert first.tolist() == [2.0, -4.0, 18.0, 0.0] and first.requires_grad
    second, = torch.autograd.grad(first @ torch.tensor([1.0, 10.0, 100.0, 1000.0], device="cuda"), t)
    assert second.tolist() == [2.0, 20.0, 600.0, 0.0]


@pytest.mark.parametrize("out_dtype", ["float32", "bfloat16"])
def test_outputs_given_by_the_caller(out_dtype):
    """A result in `out` is recorded as torch's operations in place are; what the sums were added to gets its gradient too."""
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, out_dtype)
    table, ids, w = _inputs(50, 6, 9, torch.float32, torch.int32)
    ref = table.double().requires_grad_()
    _reference(ref, ids, 2.0).backward(w.double())
    leaf = table.clone().requires_grad_()
    out = torch.empty((50, 9), dtype=dt, device="cuda")
    assert M.mlip_embed(leaf, ids, 2.0, out=out) is out and out.requires_grad
    out.backward(w.to(dt))
    assert leaf.grad.dtype == torch.float32 and torch.equal(leaf.grad, ref.grad.float())
    lost = torch.ones((50, 9), dtype=dt, device="cuda", requires_grad=True)
    M.mlip_embed(table, ids, out=lost * 1.0).backward(w.to(dt))
    assert (lost.grad == 0).all()
    part = torch.zeros((50, 12), dtype=dt, device="cuda")
    leaf.grad = None
    M.mlip_embed(leaf, ids, 2.0, out=part[:, 2:11])
    part.backward(torch.nn.functional.pad(w.to(dt), (2, 1), value=5.0))
    assert torch.equal(leaf.grad, ref.grad.float())

    g, old = w.clone().requires_grad_(), torch.ones((6, 9), dtype=dt, device="cuda", requires_grad=True)
    bar = torch.full((6, 9), 2.0, dtype=dt, device="cuda")
    for accumulate in (True, False):
        g.grad = old.grad = None
        held = old * 1.0
        assert M.mlip_embed_grad(g, ids, 6, 0.5, out=held, accumulate=accumulate) is held
        want = torch.zeros((6, 9), dtype=torch.float64, device="cuda").index_add(0, ids.long().clamp(min=0), torch.where((ids >= 0)[:, None], w.double(), 0.0))
        assert torch.equal(held.detach(), (want * 0.5 + (1.0 if accumulate else 0.0)).to(dt))
        held.backward(bar)
        assert torch.equal(g.grad, torch.where((ids >= 0)[:, None], 1.0, 0.0).expand(50, 9))
        assert torch.equal(old.grad, bar if accumulate else torch.zeros_like(bar))
        g.grad = old.grad = None
        held = torch.nn.functional.pad(old, (1, 2))
        M.mlip_embed_grad(g, ids, 6, 0.5, out=held[:, 1:10], accumulate=accumulate)
        held.backward(torch.full((6, 12), 2.0, dtype=dt, device="cuda"))
        assert torch.equal(g.grad, torch.where((ids >= 0)[:, None], 1.0, 0.0).expand(50, 9))
        assert torch.equal(old.grad, bar if accumulate else torch.zeros_like(bar))


def test_nothing_is_recorded_where_nothing_asks_for_it():
    import torch
    import paper_2506_02023_amd as M
    table, ids, w = _inputs(50, 6, 9, torch.float32, torch.int32)
    leaf = table.clone().requires_grad_()
    with torch.no_grad():
        assert not M.mlip_embed(leaf, ids).requires_grad and not M.mlip_embed_grad(w.clone().requires_grad_(), ids, 6).requires_grad
    assert not M.mlip_embed(table, ids).requires_grad and not M.mlip_embed_grad(w, ids, 6).requires_grad
