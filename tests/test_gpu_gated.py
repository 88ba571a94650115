"""Gated projections and their gradient against 64-bit arithmetic.

Tolerances count roundings: a product of fp32 accuracy over K terms is off by at most 2 (K + 8) 2^-24 times the sum of the terms' sizes, the activations
by 2^-18 of the size of what they multiply, and every rounding to the arrays' type by half a step, finfo.eps / 2."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ACTS = ["silu", "gelu", "sigmoid", "silu_sigmoid"]
U24 = 2.0 ** -24


def _make(n, d, f, dtype, bias=True, seed=0, turned=False, gap=0):
    import torch
    rng = np.random.default_rng([n, d, f, seed])

    def t(shape, std):
        return torch.as_tensor(rng.normal(size=shape) * std, dtype=dtype, device="cuda")
    x, bar = t((n, d + gap), 1.0)[:, :d], t((n, f + gap), 0.3)[:, :f]
    w = [t((f, d), d ** -0.5).t() if turned else t((d, f), d ** -0.5) for _ in range(2)]
    b = [t(f, 0.3) if bias else None for _ in range(2)]
    return bar, (x, *w, *b)


def _phi(act, g, v):
    import torch
    if act == "gelu":
        return g * torch.special.ndtr(g) * v
    s = torch.sigmoid(g)
    return {"silu": g * s * v, "sigmoid": s * v, "silu_sigmoid": s * v * torch.sigmoid(v)}[act]


def _reference(bar, inputs, act):
    """(h, its tolerance, gradients, their tolerances) without the last rounding"""
    import torch
    leaves = [None if t is None else t.detach().double().requires_grad_() for t in inputs]
    x, wg, wv, bg, bv = leaves
    g, v = x @ wg + (0 if bg is None else bg), x @ wv + (0 if bv is None else bv)
    h = _phi(act, g, v)
    u = torch.finfo(inputs[0].dtype).eps / 2
    H = bar.double()
    G, V = torch.autograd.grad(h, [g, v], H, retain_graph=True)
    grads = torch.autograd.grad(h, [t for t in leaves if t is not None], H)
    grads = [grads[k] for k in range(3)] + (list(grads[3:]) if bg is not None else [None, None])
    with torch.no_grad():
        d, n, f = x.shape[1], x.shape[0], g.shape[1]
        eg, ev = (2 * (d + 8) * U24 * (x.abs() @ w.abs() + (0 if b is None else b.abs())) for w, b in ((wg, bg), (wv, bv)))
        tol_h = 2 * (1 + v.abs() + g.abs()) * (eg + ev) + 2.0 ** -18 * (1 + g.abs()) * v.abs()
        e = H.abs() * (2 * (1 + g.abs()) * (1 + v.abs()) * (eg + ev) + 2.0 ** -18 * (1 + g.abs()) * (1 + v.abs()))
        eG, eV = e + u * G.abs(), e + u * V.abs()
        tol = [eG @ wg.abs().t() + eV @ wv.abs().t() + 2 * (2 * f + 8) * U24 * (G.abs() @ wg.abs().t() + V.abs() @ wv.abs().t())]
        tol += [x.abs().t() @ E + 2 * (n + 8) * U24 * (x.abs().t() @ Q.abs()) for E, Q in ((eG, G), (eV, V))]
        tol += [E.sum(0) + 2 * (n + 8) * U24 * Q.abs().sum(0) for E, Q in ((eG, G), (eV, V))]
    return h.detach(), tol_h, grads, tol


def _check(got, want, tol, what):
    import torch
    u = torch.finfo(got.dtype).eps / 2
    off = (got.double() - want).abs() - (tol * (1 + u) + u * want.abs() + torch.finfo(got.dtype).smallest_normal * u * 2)
    assert bool((off <= 0).all()), f"{what}: beyond its tolerance by {float(off.max()):.3e}"


def _both(n, d, f, dtype, act, **k):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    bar, inputs = _make(n, d, f, dt, **k)
    h, tol_h, grads, tol = _reference(bar, inputs, act)
    got = M.mlip_gated(*inputs, act=act)
    assert got.dtype == dt and got.shape == (n, f)
    _check(got, h, tol_h, "h")
    back = M.mlip_gated_grad(bar, *inputs, act=act)
    for name, a, b, t in zip(("dx", "dwg", "dwv", "dbg", "dbv"), back, grads, tol):
        assert (a is None) == (b is None), name
        if a is not None:
            assert a.dtype == dt
            _check(a, b, t, name)


SIZES = [(1, 1, 1), (1, 64, 128), (3, 5, 7), (108, 64, 128), (129, 64, 33), (500, 64, 256), (257, 63, 65), (200, 130, 31), (1000, 32, 96), (300, 192, 160),
         (70, 341, 100), (130, 1024, 96), (64, 96, 1365), (2500, 65, 64)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,d,f", SIZES)
def test_sizes(n, d, f, dtype):
    _both(n, d, f, dtype, ACTS[(n + d + f) % 4], bias=(n + d) % 2 == 0)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_acts(act, dtype):
    _both(333, 64, 70, dtype, act)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("gap", [1, 8])
def test_layouts(dtype, turned, gap):
    _both(190, 64, 72, dtype, "silu", turned=turned, gap=gap)
    _both(190, 128, 72, dtype, "silu", turned=turned, gap=gap)


@pytest.mark.parametrize("n,d,f", [(1024, 129, 33), (1100, 200, 100), (1030, 1025, 40), (1500, 2050, 64), (1200, 300, 700), (3000, 256, 600)])
@pytest.mark.parametrize("turned", [False, True])
def test_wide_fp32_rows(n, d, f, turned):
    """(the terms that two parts of 22 bits leave out are below 12 2^-24 of the terms' sizes, of 2 (d + 8) 2^-24 counted)"""
    _both(n, d, f, "float32", ACTS[(n + d) % 4], turned=turned, gap=(n + f) % 3, bias=n % 4 == 0)


@pytest.mark.parametrize("d", [160, 128, 61])
def test_fp32_rows_of_all_sizes(d):
    """Rows from 2^-90 to 2^122 and columns from 2^-32 to 2^31, some of them zero or not finite: each as exact as if it were alone"""
    import torch
    import paper_2506_02023_amd as M
    bar, (x, wg, wv, _, _) = _make(1100, d, 64, torch.float32, bias=False)
    x = x * torch.exp2(torch.arange(1100, device="cuda") % 213 - 90.0)[:, None]
    wv = wv * torch.exp2(torch.arange(64, device="cuda") - 32.0)[None, :]
    wv[:, 40:] *= torch.exp2(torch.tensor(-90.0, device="cuda"))      # (columns from 2^-82 on)
    x[5], wv[:, 7] = 0.0, 0.0
    h, tol, _, _ = _reference(bar, (x, wg, wv, None, None), "sigmoid")
    got = M.mlip_gated(x, wg, wv, act="sigmoid")
    # v itself has to be an fp32 number: with rows of 2^122, columns of 2^31 and d terms it reaches 2^153 and more, beyond 2^128 it is infinite in fp32 and sigmoid(g) = 0 times it NaN
    fits = (x.double() @ wv.double()).abs() < 2.0 ** 126
    _check(torch.where(fits, got, 0.0), torch.where(fits, h, 0.0), tol + 2.0 ** -140, "h")      # (what is below the normal numbers may go to zero)
    assert bool(fits[:, :30].double().mean() > 0.5) and bool(fits[:, 40:].all())
    assert bool((got[5] == 0).all()) and bool((got[:, 7] == 0).all())
    x2 = x.clone()
    x2[17, 3], x2[1099, d - 1] = float("nan"), float("inf")
    got2 = M.mlip_gated(x2, wg, wv, act="sigmoid")
    keep = torch.ones(1100, dtype=torch.bool, device="cuda")
    keep[[17, 1099]] = False
    same = keep[:, None] & fits        # (0 times infinity, elsewhere, is not equal to itself)
    assert torch.equal(got2[same], got[same]) and got2[17].isnan().all() and got2[1099].isnan().all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_rows(dtype):
    _both(50_001 if dtype == "float32" else 70_001, 64, 512 if dtype == "float32" else 1024, dtype, "silu")


def test_several_chunks():
    """More rows than a chunk has (4 GB of parts): gradients of whole numbers, all sums exact, against those of the two halves, which are one chunk each.
    (sigmoid(0) = 1/2; with x, H in -1 .. 1 and |v| <= 128 every sum is a multiple of 1/4 below 2^22.)"""
    import torch
    import paper_2506_02023_amd as M
    n, d, f = 100_000, 64, 4096
    g = torch.Generator(device="cuda").manual_seed(3)

    def whole(low, high, *shape):
        return torch.randint(low, high + 1, shape, generator=g, device="cuda").float()
    x, bar, wv, wg = whole(-1, 1, n, d), whole(-1, 1, n, f), whole(-2, 2, d, f), torch.zeros(d, f, device="cuda")
    bias = torch.zeros(f, device="cuda")
    assert n * (2 * f + d) * 6 > 4 << 30 > n // 2 * (2 * f + 128) * 6
    dx, *dw = M.mlip_gated_grad(bar, x, wg, wv, bias, bias, act="sigmoid")
    halves = [M.mlip_gated_grad(bar[k], x[k], wg, wv, bias, bias, act="sigmoid") for k in (slice(0, n // 2), slice(n // 2, n))]
    assert torch.equal(dx, torch.cat([h[0] for h in halves]))
    for k, w in enumerate(dw):
        assert torch.equal(w, halves[0][k + 1] + halves[1][k + 1]) and bool((w != 0).any())


@pytest.mark.parametrize("n,d,f,dtype", [(4100, 640, 1100, "bfloat16"), (4097, 513, 1025, "float16"), (8200, 530, 530, "float32"), (600, 1030, 300, "bfloat16")])
def test_large_tiles(n, d, f, dtype):
    _both(n, d, f, dtype, "gelu", bias=n != 4100, gap=n % 2)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_rows(dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    bar, inputs = _make(0, 64, 40, dt)
    assert M.mlip_gated(*inputs).shape == (0, 40)
    dx, *d = M.mlip_gated_grad(bar, *inputs)
    assert dx.shape == (0, 64) and all(bool((t == 0).all()) and t.shape == i.shape for t, i in zip(d, inputs[1:]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_odd_strides_and_broadcast(dtype):
    """Every second column of x, weights of any order, a gradient that is the same for all"""
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    bar, (x, wg, wv, bg, bv) = _make(70, 64, 48, dt)
    wide = torch.full((70, 128), float("nan"), dtype=dt, device="cuda")
    wide[:, ::2] = x
    w2 = torch.full((48, 2, 64), float("nan"), dtype=dt, device="cuda")
    w2[:, 1] = wv.t()
    same = M.mlip_gated(x, wg, wv, bg, bv)
    assert torch.equal(M.mlip_gated(wide[:, ::2], wg, w2[:, 1].t(), bg, bv), same)
    one = torch.full((1, 1), 0.5, dtype=dt, device="cuda").expand(70, 48)
    for a, b in zip(M.mlip_gated_grad(one, wide[:, ::2], wg, w2[:, 1].t(), bg, bv), M.mlip_gated_grad(one.contiguous(), x, wg, wv, bg, bv)):
        assert torch.equal(a, b)
    same_x = x[:1].expand(70, 64)
    assert torch.equal(M.mlip_gated(same_x, wg, wv, bg, bv), M.mlip_gated(same_x.contiguous(), wg, wv, bg, bv))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gap", [0, 1])
def test_values_that_are_not_finite_stay_in_their_row(dtype, gap):
    import torch
    import paper_2506_02023_amd as M
    bar, (x, *w) = _make(300, 64, 40, getattr(torch, dtype), gap=gap)
    clean, x2 = M.mlip_gated(x, *w), x.clone()
    x2[17, 3], x2[299, 63] = float("nan"), float("inf")
    got = M.mlip_gated(x2, *w)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[17, 299]] = False
    assert torch.equal(got[keep], clean[keep]) and got[17].isnan().all() and not got[299].isfinite().all()
    dx, dx2 = M.mlip_gated_grad(bar, x, *w)[0], M.mlip_gated_grad(bar, x2, *w)[0]
    assert torch.equal(dx2[keep], dx[keep]) and dx2[17].isnan().all()


def test_what_lies_around_outputs_and_inputs():
    """Through the C interface: places between the rows of outputs stay, places between the rows of inputs (NaN) are not used"""
    import torch
    from paper_2506_02023_amd import binding as B
    L = B.lib()
    for dtype, dt in ((0, torch.float32), (1, torch.bfloat16)):
        bar, (x, wg, wv, bg, bv) = _make(203, 64, 37, dt)

        def cut(t, gap):
            w = torch.full((t.shape[0], t.shape[1] + gap), float("nan"), dtype=dt, device="cuda")
            w[:, :t.shape[1]] = t
            return w[:, :t.shape[1]]
        bx, bb = cut(x, 8), cut(bar, 3)
        call = B._Gated(dtype, 0, 203, 64, 37, bx.data_ptr(), *bx.stride(), wg.data_ptr(), *wg.stride(), wv.data_ptr(), *wv.stride(), bg.data_ptr(), bv.data_ptr())
        out, dx = (torch.full((203, c), 7.0, dtype=dt, device="cuda") for c in (40, 70))
        need = max(L.mlip_gated_workspace(call, 0), L.mlip_gated_workspace(call, 1))
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
        assert L.mlip_gated(call, out.data_ptr(), 40, ws.data_ptr(), need, B._stream()) == 0
        g = B._GatedGrad(bb.data_ptr(), *bb.stride(), dx.data_ptr(), 70)
        ws.fill_(0xff)
        assert L.mlip_gated_grad(call, g, ws.data_ptr(), need, B._stream()) == 0
        assert torch.equal(out[:, :37], B.mlip_gated(x, wg, wv, bg, bv)) and bool((out[:, 37:] == 7).all())
        assert torch.equal(dx[:, :64], B.mlip_gated_grad(bar, x, wg, wv, bg, bv)[0]) and bool((dx[:, 64:] == 7).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_autograd_and_differences(dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    bar, inputs = _make(50, 33, 20, dt, turned=True)
    leaves = [t.detach().clone().requires_grad_() for t in inputs]
    out = M.mlip_gated(*leaves, act="gelu")
    out.backward(bar)
    for leaf, want in zip(leaves, M.mlip_gated_grad(bar, *inputs, act="gelu")):
        assert torch.equal(leaf.grad, want)
    only = [t.detach() for t in inputs]
    only[2] = only[2].clone().requires_grad_()
    M.mlip_gated(*only, act="gelu").backward(bar)
    assert torch.equal(only[2].grad, leaves[2].grad)
    if dtype == "float32":     # central differences along a direction: error h^2 of the third derivative and 2^-24 / h of the values
        h = 2.0 ** -6
        for k, leaf in enumerate(leaves):
            way = torch.randn(leaf.shape, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda")
            way = way / way.norm()

            def value(s):
                moved = [t.detach().double() for t in inputs]
                moved[k] = moved[k] + s * way.double()
                g, v = moved[0] @ moved[1] + moved[3], moved[0] @ moved[2] + moved[4]
                return float((_phi("gelu", g, v) * bar.double()).sum())
            slope = (value(h) - value(-h)) / (2 * h)
            assert abs(slope - float((leaf.grad.double() * way.double()).sum())) <= 2e-3 * float(leaf.grad.norm()) + 1e-4


def test_second_derivatives_are_refused():
    import torch
    import paper_2506_02023_amd as M
    _, inputs = _make(8, 8, 8, torch.float32)
    x = inputs[0].clone().requires_grad_()
    d, = torch.autograd.grad(M.mlip_gated(x, *inputs[1:]).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_captured_and_on_other_streams(dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    bar, inputs = _make(700, 64, 100, dt)
    x = inputs[0].clone()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        M.mlip_gated(x, *inputs[1:])
        M.mlip_gated_grad(bar, x, *inputs[1:])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = M.mlip_gated(x, *inputs[1:])
        d = M.mlip_gated_grad(bar, x, *inputs[1:])
    for k in range(4):
        x.copy_(_make(700, 64, 100, dt, seed=k + 1)[1][0])
        graph.replay()
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            want = M.mlip_gated(x, *inputs[1:]), *M.mlip_gated_grad(bar, x, *inputs[1:])
        torch.cuda.synchronize()
        for a, b in zip((h, *d), want):
            assert torch.equal(a, b)
