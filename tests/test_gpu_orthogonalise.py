"""Orthogonal updates against the same iteration in 64 bits.

Tolerance, in the norm of all elements: a step's result is off by 2^-18 |X_k| at most (parts of 22 bits: three roundings of 2^-22 of sizes up to
|a| + |b| + |c| = 10.3 times |X_k|, and fp32 sums), later steps stretch that by a = 3.4445 at most each, and the last rounding adds half a step.  Of bf16
matrices the products take parts of 11 bits; what that brings (0.4 to 1.2e-3 of the norm) and the 1.7e-3 of the result's own rounding together
lie within the half step of 3.9e-3 that is counted for the latter."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)


def _make(rows, cols, dtype, seed=0, kind="lowrank"):
    import torch
    rng = np.random.default_rng([rows, cols, seed])
    m = rng.normal(size=(rows, cols)) * 0.3
    if kind == "lowrank":
        r = max(1, min(rows, cols) // 8)
        m += rng.normal(size=(rows, r)) @ rng.normal(size=(r, cols)) / r ** 0.5
    return torch.as_tensor(m * 1e-3, dtype=dtype, device="cuda")


def _reference(g, steps=5, coef=COEF, eps=1e-7, scale=1.0):
    """(result, tolerance of the norm of the difference, without the last rounding)"""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / max(float(x.norm()), eps)
    a, b, c = coef
    tol = 2.0 ** -20 * float(x.norm())
    for _ in range(steps):
        p = x @ x.t()
        tol = a * tol + 2.0 ** -18 * float(x.norm())
        x = a * x + (b * p + c * (p @ p)) @ x
    return scale * (x.t() if tall else x), abs(scale) * tol


def _check(got, g, what="", **k):
    import torch
    want, tol = _reference(g, **k)
    assert got.dtype == g.dtype and got.shape == g.shape
    off, u = float((got.double() - want).norm()), torch.finfo(got.dtype).eps / 2
    assert off <= tol * (1 + u) + u * float(want.norm()) * 1.001 + 1e-30, f"{what} {tuple(g.shape)}: off by {off:.3e} of {float(want.norm()):.3e}, tolerance {tol:.3e}"


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 200), (8, 64), (64, 8), (63, 65), (64, 64), (64, 128), (128, 64), (65, 129), (127, 127), (128, 128), (130, 40), (200, 333),
          (256, 256), (129, 1000), (1000, 129), (300, 2000), (512, 700), (700, 700), (1024, 1500)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_shapes_one_by_one(dtype):
    import torch
    import paper_2506_02023_amd as M
    for shape in SHAPES:
        g = _make(*shape, getattr(torch, dtype))
        out = torch.full_like(g, 7.0)
        assert M.mlip_orthogonalise([g], out=[out])[0] is out
        _check(out, g)


def test_a_list_of_all_shapes_and_types():
    """More matrices than a launch takes, and those of each the same bits as alone"""
    import torch
    import paper_2506_02023_amd as M
    dts = [torch.float32, torch.bfloat16, torch.float16]
    list_ = [_make(*s, dts[k % 3], seed=k // len(SHAPES)) for k, s in enumerate(SHAPES * 2)] + [torch.empty(0, 5, device="cuda"), torch.empty(4, 0, device="cuda")]
    copies = [t.clone() for t in list_]
    res = M.mlip_orthogonalise(list_)
    for k, (t, g, r) in enumerate(zip(list_, copies, res)):
        assert r is t
        if t.numel():
            _check(t, g, k)
            assert torch.equal(M.mlip_orthogonalise([g.clone()])[0], t)
    assert M.mlip_orthogonalise([]) == []


def test_matrices_beyond_the_scratch_memory_of_a_group():
    """Four matrices of 560 MB of scratch memory each are taken in two groups: the same bits as alone"""
    import torch
    import paper_2506_02023_amd as M
    from paper_2506_02023_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(1)
    list_ = [torch.randn(5000, 9000, generator=g, device="cuda") for _ in range(4)]
    a = (B._Matrix * 4)(*[B._Matrix(t.data_ptr(), t.data_ptr(), *t.shape, *t.stride(), *t.stride(), 0) for t in list_])
    assert 1 << 30 < B.lib().mlip_orthogonalise_workspace(a, 4) <= 1 << 31
    alone = [M.mlip_orthogonalise([t], steps=2, out=[torch.empty_like(t)])[0] for t in list_]
    assert all(torch.equal(x, y) for x, y in zip(M.mlip_orthogonalise(list_, steps=2), alone))


def test_singular_values():
    """They end between 0.67 and 1.21 where they began above 0.003 of the norm (the interval that five steps of these coefficients reach)"""
    import torch
    import paper_2506_02023_amd as M
    g = _make(200, 300, torch.float32)
    s0 = torch.linalg.svdvals(g.double().cpu())
    assert float(s0[-1] / s0.square().sum().sqrt()) > 0.003
    s = torch.linalg.svdvals(M.mlip_orthogonalise([g])[0].double().cpu())
    assert 0.67 < float(s.min()) and float(s.max()) < 1.21


@pytest.mark.parametrize("shape", [(40, 70), (300, 200), (130, 1000)])
@pytest.mark.parametrize("steps,coef,scale", [(0, COEF, 2.0), (1, COEF, 1.0), (3, (1.5, -0.5, 0.0), 0.2), (12, (1.875, -1.25, 0.375), -1.0), (8, COEF, 1.0)])
def test_steps_coefficients_scale(shape, steps, coef, scale):
    import torch
    import paper_2506_02023_amd as M
    g = _make(*shape, torch.float32)
    got = M.mlip_orthogonalise([g.clone()], steps=steps, coefficients=coef, scale=scale)[0]
    _check(got, g, steps=steps, coef=coef, scale=scale)


def test_sizes_of_gradients():
    """Tiny, large and zero gradients; eps takes over below it"""
    import torch
    import paper_2506_02023_amd as M
    for shape in ((40, 50), (300, 200)):
        g = _make(*shape, torch.float32)
        one = M.mlip_orthogonalise([g.clone()], eps=0.0)[0]
        for f in (2.0 ** -90, 2.0 ** 80):
            assert torch.equal(M.mlip_orthogonalise([g * f], eps=0.0)[0], one)
        small = g / g.norm() * 1e-9
        _check(M.mlip_orthogonalise([small.clone()], eps=1e-7)[0], small, eps=1e-7)
        for eps, steps in ((1e-7, 5), (0.0, 5), (0.0, 0)):
            assert bool((M.mlip_orthogonalise([torch.zeros(shape, device="cuda")], eps=eps, steps=steps)[0] == 0).all())


def test_decaying_singular_values():
    """What is 10^-5 of the largest singular value is stretched by 485 and has to come out of its roundings"""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(5)
    for m, n in ((100, 100), (200, 500)):
        u, v = np.linalg.qr(rng.normal(size=(m, m)))[0], np.linalg.qr(rng.normal(size=(n, m)))[0]
        g = torch.as_tensor(u * np.logspace(0, -5, m) @ v.T, dtype=torch.float32, device="cuda")
        _check(M.mlip_orthogonalise([g.clone()])[0], g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layouts_and_stacks(dtype):
    """Transposed, cut out, strided and stacked matrices: the same bits as of their copies; places around them stay"""
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    for shape in ((50, 90), (150, 333)):
        g = _make(*shape, dt)
        want = M.mlip_orthogonalise([g.clone()])[0]
        assert torch.equal(M.mlip_orthogonalise([g.t().contiguous().t()])[0], want)
        wide = torch.full((shape[0], 2 * shape[1] + 3), 7.0, dtype=dt, device="cuda")
        wide[:, 1:2 * shape[1]:2] = g
        M.mlip_orthogonalise([wide[:, 1:2 * shape[1]:2]])
        assert torch.equal(wide[:, 1:2 * shape[1]:2], want) and bool((wide[:, ::2] == 7).all()) and bool((wide[:, -2:] == 7).all())
        stack = torch.stack([g, _make(*shape, dt, seed=1), g])
        M.mlip_orthogonalise([stack])
        assert torch.equal(stack[0], want) and torch.equal(stack[2], want)
        out = torch.empty_like(stack).transpose(1, 2).contiguous().transpose(1, 2)
        M.mlip_orthogonalise([torch.stack([g, g, g])], out=[out])
        assert torch.equal(out[1], want)


def test_values_that_are_not_finite_stay_in_their_matrix():
    import torch
    import paper_2506_02023_amd as M
    for shape in ((40, 60), (200, 300)):
        a, b = _make(*shape, torch.float32), _make(*shape, torch.float32, seed=1)
        want = M.mlip_orthogonalise([a.clone()])[0]
        for bad in (float("nan"), float("inf"), -float("inf")):
            b[7, 9] = bad
            c = a.clone()
            out = M.mlip_orthogonalise([b.clone(), c])
            assert torch.equal(out[1], want) and not bool(out[0].isfinite().any())


def test_captured_and_on_other_streams():
    import torch
    import paper_2506_02023_amd as M
    src = [_make(*s, torch.float32) for s in ((64, 64), (200, 300), (30, 700))]
    out = [torch.empty_like(t) for t in src]
    M.mlip_orthogonalise(src, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mlip_orthogonalise(src, out=out)
    stream = torch.cuda.Stream()
    for k in range(4):
        for t in src:
            t.copy_(_make(*t.shape, torch.float32, seed=k + 1))
        graph.replay()
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            want = M.mlip_orthogonalise([t.clone() for t in src])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_versions():
    """What the call writes is known to autograd as written"""
    import torch
    import paper_2506_02023_amd as M
    t = _make(8, 8, torch.float32)
    before = t._version
    M.mlip_orthogonalise([t])
    assert t._version > before
