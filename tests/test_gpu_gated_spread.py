"""Gated projections of fp32 rows and columns whose values span many powers of two, where small ones meet large ones, against 64-bit arithmetic.

Tolerances are those of test_gpu_gated.py: fp32 accuracy, 2 (d + 8) 2^-24 of the sum of the terms' sizes |x_i| |W_ic|, whatever the spread."""
import pytest

from test_gpu_gated import _check, _make, _reference

pytestmark = pytest.mark.gpu

INPUTS = ("x", "wg", "wv", "bg", "bv")


def _compare(bar, inputs, act, grads=True):
    import paper_2506_02023_amd as M
    h, tol_h, want, tol = _reference(bar, inputs, act)
    _check(M.mlip_gated(*inputs, act=act), h, tol_h, "h")
    if grads:
        for name, a, b, t in zip(INPUTS, M.mlip_gated_grad(bar, *inputs, act=act), want, tol):
            if a is not None:
                _check(a, b, t, "d" + name)


@pytest.mark.parametrize("spread", [18, 22, 24, 32, 40, 80])
@pytest.mark.parametrize("n,d,f", [(108, 64, 40), (300, 128, 70), (90, 17, 33), (1023, 160, 40), (1024, 160, 40), (1100, 600, 300), (1500, 700, 512), (4000, 260, 490)])
def test_small_features_with_large_weights(n, d, f, spread):
    """Every second feature is 2^spread smaller than the others, and its weights larger by as much: all terms of a sum are of one size"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
    by = torch.where(torch.arange(d, device="cuda") % 2 == 0, 2.0 ** (spread // 2), 2.0 ** (spread // 2 - spread))
    _compare(bar, (x * by, wg / by[:, None], wv / by[:, None], bg, bv), "silu")


@pytest.mark.parametrize("n,d,f", [(200, 64, 96), (1100, 192, 96), (1030, 1000, 501)])
@pytest.mark.parametrize("order", ["rows", "columns"])
def test_features_that_only_some_columns_use(n, d, f, order):
    """Blocks of weights, zeros between them: what a column does not use may be 2^50 times what it does ("rows": the features, "columns": the weights)"""
    import torch
    bar, (x, wg, wv, _, _) = _make(n, d, f, torch.float32)
    block = (torch.arange(d, device="cuda")[:, None] * 3 // d) == (torch.arange(f, device="cuda")[None, :] * 3 // f)
    size = torch.exp2(25.0 * (torch.arange(d, device="cuda") * 3 // d - 1))
    if order == "rows":
        _compare(bar, (x * size, wg * block / size[:, None], wv * block / size[:, None], None, None), "sigmoid")
    else:       # rows of x that use one block of features each, of weights that differ by 2^50
        mine = (torch.arange(n, device="cuda")[:, None] % 3) == (torch.arange(d, device="cuda")[None, :] * 3 // d)
        _compare(bar, (x * mine / size, wg * size[:, None], wv * size[:, None], None, None), "sigmoid")


@pytest.mark.parametrize("n,d,f", [(500, 96, 64), (2000, 300, 64), (2000, 512, 500)])
def test_rows_with_one_large_feature(n, d, f):
    """One feature of every row 2^30 times the others, with weights of zero in half of the columns; one-hot rows and rows of zeros among them"""
    import torch
    bar, (x, wg, wv, _, _) = _make(n, d, f, torch.float32)
    x = x.clone()
    x[:, 5] *= 2.0 ** 30
    x[::7] = torch.nn.functional.one_hot(torch.arange(n, device="cuda") % d, d).float()[::7]
    x[3], x[n - 1] = 0.0, 0.0
    wg, wv = wg.clone(), wv.clone()
    wg[5, ::2], wv[5, ::2] = 0.0, 0.0
    wg[5, 1::2], wv[5, 1::2] = 2.0 ** -31, 2.0 ** -30
    wg[:, 8] = 0.0
    _compare(bar, (x, wg, wv, None, None), "silu_sigmoid")


@pytest.mark.parametrize("n,d,f", [(300, 64, 72), (1100, 160, 72), (3001, 300, 600)])
def test_rows_are_alone(n, d, f):
    """The same bits for a row and column whatever lies beside them: in a batch with rows and columns of great spread, and without"""
    import torch
    import paper_2506_02023_amd as M
    _, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
    x2, wv2 = x.clone(), wv.clone()
    by = torch.exp2(torch.arange(d, device="cuda") % 2 * 40.0)
    x2[10::11] *= by
    wv2[:, 6::9] /= by[:, None]
    one, two = M.mlip_gated(x, wg, wv, bg, bv), M.mlip_gated(x2, wg, wv2, bg, bv)
    rows, cols = torch.arange(n, device="cuda") % 11 != 10, torch.arange(f, device="cuda") % 9 != 6
    assert torch.equal(one[rows][:, cols], two[rows][:, cols]) and not torch.equal(one, two)


@pytest.mark.parametrize("n,d,f", [(300, 64, 72), (1100, 160, 72), (3001, 300, 600)])
def test_strides_do_not_matter(n, d, f):
    """Rows and columns of great spread in other layouts: the same bits"""
    import torch
    import paper_2506_02023_amd as M
    _, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
    by = torch.exp2(torch.arange(d, device="cuda") % 2 * 40.0)
    x, wg, wv = x * by, wg / by[:, None], wv / by[:, None]
    want = M.mlip_gated(x, wg, wv, bg, bv)
    assert torch.equal(M.mlip_gated(x.t().contiguous().t(), wg.t().contiguous().t(), wv, bg, bv), want)
    wide = torch.full((d, 2 * f), float("nan"), device="cuda")
    wide[:, ::2] = wv
    assert torch.equal(M.mlip_gated(x, wg, wide[:, ::2], bg, bv), want)


@pytest.mark.parametrize("n,d,f", [(300, 64, 72), (300, 160, 72), (3001, 300, 600)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_weights_that_are_not_finite_stay_in_their_column(n, d, f, dtype):
    import torch
    import paper_2506_02023_amd as M
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, getattr(torch, dtype))
    clean, back = M.mlip_gated(x, wg, wv, bg, bv), M.mlip_gated_grad(bar, x, wg, wv, bg, bv)
    wg2, wv2 = wg.clone(), wv.clone()
    wg2[3, 9], wv2[d - 1, 40], wv2[0, 71] = float("nan"), float("inf"), float("nan")
    got, back2 = M.mlip_gated(x, wg2, wv2, bg, bv), M.mlip_gated_grad(bar, x, wg2, wv2, bg, bv)
    keep = torch.ones(f, dtype=torch.bool, device="cuda")
    keep[[9, 40, 71]] = False
    assert torch.equal(got[:, keep], clean[:, keep]) and got[:, [9, 71]].isnan().all() and not got[:, 40].isfinite().any()
    for a, b in zip(back[1:], back2[1:]):
        assert torch.equal(a[..., keep], b[..., keep])


@pytest.mark.parametrize("n,d,f", [(1100, 64, 48), (1100, 160, 48), (3001, 300, 600)])
def test_rows_and_columns_of_tiny_values(n, d, f):
    """Rows down to 2^-120 of the usual size and columns that bring their results back: as exact as others"""
    import torch
    bar, (x, wg, wv, _, _) = _make(n, d, f, torch.float32)
    x = x * torch.exp2(-(torch.arange(n, device="cuda") % 121.0))[:, None]
    _compare(bar, (x, wg * 2.0 ** 40, wv * 2.0 ** 60, None, None), "sigmoid", grads=False)


@pytest.mark.parametrize("n,d,f", [(1024, 1025, 480), (2100, 500, 700), (1000, 2050, 260), (6000, 200, 420)])
@pytest.mark.parametrize("turned", [False, True])
def test_wide_rows(n, d, f, turned):
    """Sizes of n d f >= 5e8, which go by scaled parts, in other layouts; the terms that two parts of 22 bits leave out are below 12 2^-24 of the terms' sizes"""
    import torch
    bar, inputs = _make(n, d, f, torch.float32, turned=turned, gap=n % 3, bias=n % 4 == 0)
    assert n * d * f >= 5e8
    _compare(bar, inputs, ["silu", "gelu", "sigmoid", "silu_sigmoid"][(n + d) % 4], grads=False)


@pytest.mark.parametrize("n,d,f", [(3001, 300, 600), (500, 61, 64)])
def test_rows_of_all_sizes(n, d, f):
    """Rows from 2^-90 to 2^60, some zero or not finite: each as exact as if it were alone"""
    import torch
    import paper_2506_02023_amd as M
    bar, (x, wg, wv, _, _) = _make(n, d, f, torch.float32)
    x = x * torch.exp2(torch.arange(n, device="cuda") % 151 - 90.0)[:, None]
    x[5], wv[:, 7] = 0.0, 0.0
    _compare(bar, (x, wg, wv, None, None), "sigmoid", grads=False)
    got, x2 = M.mlip_gated(x, wg, wv, act="sigmoid"), x.clone()
    x2[17, 3], x2[n - 1, d - 1] = float("nan"), float("inf")
    got2 = M.mlip_gated(x2, wg, wv, act="sigmoid")
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[[17, n - 1]] = False
    assert torch.equal(got2[keep], got[keep]) and got2[[17, n - 1]].isnan().all()


@pytest.mark.parametrize("n,d,f", [(200, 64, 96), (3001, 300, 600)])
def test_sparse_rows(n, d, f):
    """Rows of which nine values of ten are zero, or all but one"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
    rng = torch.Generator(device="cuda").manual_seed(n)
    x = torch.where(torch.rand(n, d, generator=rng, device="cuda") < 0.9, 0.0, x)
    x[::3] = torch.nn.functional.one_hot(torch.arange(n, device="cuda") * 7 % d, d).float()[::3] * 0.3
    _compare(bar, (x, wg, wv, bg, bv), "silu")


def test_captured():
    """Small and large spread in turn through one graph"""
    import torch
    import paper_2506_02023_amd as M
    for n, d, f in ((300, 64, 72), (3001, 300, 600)):
        bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
        by = torch.exp2(torch.arange(d, device="cuda") % 2 * 40.0)
        one, two = x.clone(), x * by
        M.mlip_gated(x, wg, wv, bg, bv)
        M.mlip_gated_grad(bar, x, wg, wv, bg, bv)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = M.mlip_gated(x, wg, wv, bg, bv), *M.mlip_gated_grad(bar, x, wg, wv, bg, bv)
        for now in (one, two, one, two):
            x.copy_(now)
            graph.replay()
            for a, b in zip(held, (M.mlip_gated(now, wg, wv, bg, bv), *M.mlip_gated_grad(bar, now, wg, wv, bg, bv))):
                assert torch.equal(a, b)
            torch.cuda.synchronize()


@pytest.mark.parametrize("n,d,f", [(300, 64, 72), (300, 128, 40)])
def test_gradients_of_strided_rows(n, d, f):
    """Great spread, every second column of x, a gradient that is one for all: the same bits as of copies"""
    import torch
    import paper_2506_02023_amd as M
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float32)
    by = torch.exp2(torch.arange(d, device="cuda") % 2 * 40.0)
    wide = torch.full((n, 2 * d), float("nan"), device="cuda")
    wide[:, 1::2] = x * by
    one = bar[:, :1].expand(n, f)
    for a, b in zip(M.mlip_gated_grad(one, wide[:, 1::2], wg, wv / by[:, None], bg, bv), M.mlip_gated_grad(one.contiguous(), x * by, wg, wv / by[:, None], bg, bv)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,d,f,dtype", [(6_000_000, 130, 32, "float32"), (12_000_000, 192, 24, "bfloat16")])
def test_rows_of_several_chunks(n, d, f, dtype):
    """More rows than 4 GB of scratch memory take: those around the ends of chunks and others as in a call of their own, some of great spread among them"""
    import torch
    import paper_2506_02023_amd as M
    from paper_2506_02023_amd import binding as B
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, d, generator=g, device="cuda", dtype=torch.float32).to(dt)
    wg, wv = ((torch.randn(d, f, generator=g, device="cuda") / d ** 0.5).to(dt) for _ in range(2))
    x[::1009, ::2] *= 2.0 ** -40
    call, _ = B._gated_call(x, wg, wv, None, None, "silu")
    need = B.lib().mlip_gated_workspace(call, 0)
    assert 4e9 < need < 4.5e9 and n * d * f > 5e8       # (a chunk's rows take all but some kilobytes of it)
    row = (d + 63) // 64 * 64
    row = (row | 64) * (4 if dtype == "float32" else 2)
    end = (4 << 30) // row // 1024 * 1024
    at = torch.cat([torch.arange(0, 3000), torch.arange(end - 4000, end + 5000), torch.arange(n - 3000, n), torch.arange(0, n, 1009)[:3000]]).cuda()
    out = M.mlip_gated(x, wg, wv)[at]
    assert len(at) * d * f < 5e8
    again = -(-int(5e8) // (len(at) * d * f)) + 1       # (as often as makes a call of the same way)
    assert torch.equal(M.mlip_gated(x[at].repeat(again, 1), wg, wv)[:len(at)], out)
