"""Gradients of gated projections of fp16 arrays at the ends of fp16's range, against 64-bit arithmetic: the gradients of g and v themselves, which the call
does not give out, may lie beyond it on either side.

Tolerances as in test_gpu_gated.py."""
import pytest

from test_gpu_gated import _check, _make, _reference

pytestmark = pytest.mark.gpu

NAMES = ("dx", "dwg", "dwv", "dbg", "dbv")


def _compare(bar, inputs, act):
    import torch
    import paper_2506_02023_amd as M
    _, _, want, tol = _reference(bar, inputs, act)
    back = M.mlip_gated_grad(bar, *inputs, act=act)
    for name, a, b, t in zip(NAMES, back, want, tol):
        if a is not None and b is not None:     # (the reference has both biases' gradients or none)
            assert bool((b.abs() < 60000).all()), f"{name} itself is beyond fp16"
            assert a.dtype == torch.float16
            _check(a, b, t, name)
    return back


@pytest.mark.parametrize("n,d,f", [(200, 64, 40), (150, 128, 96), (180, 200, 70), (600, 512, 512)])
def test_large_gradients_of_the_products(n, d, f):
    """H = 100, v about 4000 and g = 0: the gradient of g is 10^5, those of x and of the weights are up to some ten thousand"""
    import torch
    bar, (x, wg, wv, _, bv) = _make(n, d, f, torch.float16)
    bar = torch.where(bar > 0, 100.0, -100.0).half()
    rng = torch.Generator(device="cuda").manual_seed(n)
    x, wg = x * (0.05 / n ** 0.5), torch.where(torch.rand(d, f, generator=rng, device="cuda") < 0.5, 0.0, wg.float() * 1e-3).half()
    assert float((bar.double() * 0.25 * 4000).abs().max()) > 65504
    _compare(bar, (x, wg, wv, None, torch.full_like(bv, 4000.0)), "sigmoid")


@pytest.mark.parametrize("n,d,f", [(60_000, 32, 40), (20_000, 128, 64), (20_000, 200, 64), (9000, 512, 512)])
def test_small_gradients_of_many_rows(n, d, f):
    """H is 2^-23, so the gradients of g and v are below fp16's smallest number, 2^-24, and their sums are not"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float16)
    back = _compare(torch.full_like(bar, 2.0 ** -23), (x.abs(), wg, wv, bg - 2.0, bv), "sigmoid")
    assert all(bool((t != 0).double().mean() > 0.5) for t in back[1:])


@pytest.mark.parametrize("n,d,f", [(500, 64, 64), (700, 192, 96)])
def test_gradients_of_all_sizes(n, d, f):
    """H from 2^-20 to 2^8 by row, features' gates from closed to open by column"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, torch.float16)
    bar = (bar.double() * torch.exp2(torch.arange(n, device="cuda") % 29 - 20.0)[:, None]).half()
    x = (x.double() * torch.exp2(-8.0 + (-torch.arange(n, device="cuda")) % 9)[:, None]).half()
    _compare(bar, (x, wg, wv, (bg.double() + torch.linspace(-9, 3, f, device="cuda")).half(), bv), "sigmoid")
