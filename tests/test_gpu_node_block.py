"""The node network's operators together, as a fit uses them: species table, blocks of norm, gated projections and residual sum, loss by structure, clipping, updates.

One step's gradients are compared with autograd's on the same network in 64 bits, to a tolerance that counts roundings: with u half a step of the type, every operator rounds
its results once, and so does what comes back through it; 24 such roundings lie on the longest way from the loss to a weight and back, each of which is off by u of
the size of the whole at most where they add up (norm of the difference by norm of the gradient)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

N, D, F, S, BLOCKS, B = 700, 64, 96, 5, 2, 9


def _parameters(dtype):
    import torch
    rng = np.random.default_rng(11)

    def t(*shape, std=1.0, mean=0.0, dt=dtype):
        return torch.as_tensor(rng.normal(size=shape) * std + mean, dtype=dt, device="cuda")
    table, blocks = t(S, D), []
    for _ in range(BLOCKS):
        blocks.append(dict(wg=t(D, F, std=D ** -0.5), wv=t(F, D, std=D ** -0.5), down=t(F, D, std=F ** -0.5), bg=t(F, std=0.1), scale=t(D, std=0.1, mean=0.5, dt=torch.float32),
                           pre=t(D, std=0.1, mean=1.0, dt=torch.float32), post=t(D, std=0.1, mean=1.0, dt=torch.float32), gate=t(N, 1, std=0.3, mean=1.0)))
    species = torch.as_tensor(rng.integers(0, S, N), device="cuda")
    structure = torch.as_tensor(np.sort(rng.integers(0, B, N)), device="cuda", dtype=torch.int32)
    return table, blocks, species, structure, t(B, D, dt=torch.float32)


def _ours(table, blocks, species, structure):
    import paper_2506_02023_amd as M
    x = M.mlip_embed(table, species)
    y = M.mlip_norm(x, blocks[0]["pre"], kind="layer")
    for k, b in enumerate(blocks):
        h = M.mlip_gated(y, b["wg"], b["wv"].t(), b["bg"], None, "silu_sigmoid") @ b["down"]
        nxt = blocks[k + 1]["pre"] if k + 1 < BLOCKS else None
        out = M.mlip_residual(x, h, b["gate"], b["scale"], post=(b["post"], None), pre=None if nxt is None else (nxt, None), kind="layer")
        x, y = out if nxt is not None else (out, None)
    return M.mlip_embed_grad(x, structure, B, 1.0 / 16)


def _plain(table, blocks, species, structure):
    import torch

    def norm(t, w):
        t = t - t.mean(1, keepdim=True)
        return t * (t.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w
    x = table[species.long()]
    for b in blocks:
        y = norm(x, b["pre"])
        g, v = y @ b["wg"] + b["bg"], y @ b["wv"].t()
        h = (torch.sigmoid(g) * v * torch.sigmoid(v)) @ b["down"]
        x = x + b["gate"] * b["scale"] * norm(h, b["post"])
    return torch.zeros(B, D, dtype=x.dtype, device="cuda").index_add(0, structure.long(), x) / 16


def _leaves(table, blocks):
    return [table] + [b[k] for b in blocks for k in sorted(b)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_one_step(dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    table, blocks, species, structure, want = _parameters(dt)
    for leaf in _leaves(table, blocks):
        leaf.requires_grad_()
    out = _ours(table, blocks, species, structure)
    out.backward((out.detach().float() - want).to(dt))
    table64, blocks64 = table.detach().double().requires_grad_(), [{k: v.detach().double().requires_grad_() for k, v in b.items()} for b in blocks]
    out64 = _plain(table64, blocks64, species, structure)
    out64.backward((out.detach().float() - want).to(dt).double())
    u = torch.finfo(dt).eps / 2
    tol = 24 * max(u, 2.0 ** -20)      # fp32: sums of up to 700 terms, 2^-20 of their sizes
    assert float((out.detach().double() - out64).norm()) <= tol * float(out64.norm())
    for leaf, ref in zip(_leaves(table, blocks), _leaves(table64, blocks64)):
        assert leaf.grad.dtype == leaf.dtype
        assert float((leaf.grad.double() - ref.grad).norm()) <= tol * float(ref.grad.norm())

    leaves = _leaves(table, blocks)
    grads = [leaf.grad for leaf in leaves]
    norm = M.mlip_clip_grads(grads, 0.5)
    assert abs(float(norm) - float(torch.stack([r.grad.square().sum() for r in _leaves(table64, blocks64)]).sum().sqrt())) <= tol * float(norm)
    matrices = [b[k].grad for b in blocks for k in ("wg", "wv", "down")]
    before = [m.double() for m in matrices]
    updates = M.mlip_orthogonalise([m.clone() for m in matrices])
    for m, o in zip(before, updates):     # the update has the gradient's singular vectors: it points its way
        assert float((m * o.double()).sum()) > 0.67 * float(torch.linalg.svdvals(m.cpu()).sum()) * 0.5
    with torch.no_grad():
        for b, k, o in zip([b for b in blocks for _ in range(3)], ["wg", "wv", "down"] * BLOCKS, updates):
            b[k].sub_(o, alpha=1e-3)
    _ours(table, blocks, species, structure)


def test_a_step_captured():
    """Forward, backward and update in one graph, replayed on other inputs, against the same calls made one by one"""
    import torch
    import paper_2506_02023_amd as M
    table, blocks, species, structure, want = _parameters(torch.float32)
    b = blocks[0]
    x, dn = torch.randn(N, D, device="cuda"), torch.randn(N, D, device="cuda")
    weights = (b["wg"], b["wv"].t(), b["bg"], None)

    def step():
        y = M.mlip_norm(x, b["pre"])
        h = M.mlip_gated(y, *weights)
        dy, dwg, dwv, dbg, _ = M.mlip_gated_grad(h, y, *weights)
        z, n = M.mlip_residual(x, dy, b["gate"], b["scale"], post=(b["post"], None), pre=(b["pre"], None))
        back = M.mlip_residual_grad(z, dn, x, dy, b["gate"], b["scale"], post=(b["post"], None), pre=(b["pre"], None))
        dx, dw, _ = M.mlip_norm_grad(back[1], x, b["pre"])
        norm = M.mlip_clip_grads([dwg, dwv], 1.0)
        M.mlip_orthogonalise([dwg, dwv])
        return [y, h, dy, dbg, z, n, *back[:4], back[4][0], back[5][0], dx, dw, norm, dwg, dwv]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        x.normal_()
        dn.normal_()
        graph.replay()
        got = [t.clone() for t in held]
        for a, c in zip(got, step()):
            assert torch.equal(a, c)
        torch.cuda.synchronize()
