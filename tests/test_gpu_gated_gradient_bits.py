"""Gradients of gated projections of 16-bit arrays where they are sums that nearly cancel, or of equal terms, against 64-bit arithmetic.

Tolerances as in test_gpu_gated.py, with what G and V (the gradients of g and v) lose on their way into the products: two bf16 parts are off by 2^-16 of a value at most, and of fp16
arrays the product of both low parts is left out, 2^-16 of a term.  2^-15 of the terms' sizes is counted, not the half step of the arrays' type, 2^-8 or 2^-11, that those have."""
import pytest

from test_gpu_gated import U24, _check, _make, _phi

pytestmark = pytest.mark.gpu

NAMES = ("dx", "dwg", "dwv", "dbg", "dbv")


def _compare(bar, inputs, act):
    import torch
    import paper_2506_02023_amd as M
    leaves = [t.detach().double().requires_grad_() for t in inputs]
    x, wg, wv, bg, bv = leaves
    g, v = x @ wg + bg, x @ wv + bv
    h, H = _phi(act, g, v), bar.double()
    G, V = torch.autograd.grad(h, [g, v], H, retain_graph=True)
    want = torch.autograd.grad(h, leaves, H)
    with torch.no_grad():
        n, d, f = x.shape[0], x.shape[1], g.shape[1]
        eg, ev = (2 * (d + 8) * U24 * (x.abs() @ w.abs() + b.abs()) for w, b in ((wg, bg), (wv, bv)))
        e = H.abs() * (2 * (1 + g.abs()) * (1 + v.abs()) * (eg + ev) + 2.0 ** -18 * (1 + g.abs()) * (1 + v.abs()))
        eG, eV = e + 2.0 ** -15 * G.abs(), e + 2.0 ** -15 * V.abs()
        tol = [eG @ wg.abs().t() + eV @ wv.abs().t() + 2 * (2 * f + 8) * U24 * (G.abs() @ wg.abs().t() + V.abs() @ wv.abs().t())]
        tol += [x.abs().t() @ E + 2 * (n + 8) * U24 * (x.abs().t() @ Q.abs()) for E, Q in ((eG, G), (eV, V))]
        tol += [E.sum(0) + 2 * (n + 8) * U24 * Q.abs().sum(0) for E, Q in ((eG, G), (eV, V))]
    for name, a, b, t in zip(NAMES, M.mlip_gated_grad(bar, *inputs, act=act), want, tol):
        _check(a, b, t, name)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d,f", [(10, 256, 1), (435, 64, 1), (3000, 121, 1), (12, 2, 4), (15, 490, 17), (4867, 154, 19), (500, 64, 256), (700, 200, 130), (600, 512, 512), (1, 64, 64)])
def test_sums_of_both_signs(n, d, f, dtype):
    """(the sums' results are a fraction of their terms: for every second row the gradient is the one before's, the other way round, in the biases' and weights' sums)"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, getattr(torch, dtype))
    bar, x = bar.contiguous(), x.contiguous()
    if n > 1:
        x[1::2] = x[:n - n % 2:2] * (1 + 2.0 ** -6)
        bar[1::2] = -bar[:n - n % 2:2]
    _compare(bar, (x, wg, wv, bg, bv), ["silu", "gelu", "sigmoid", "silu_sigmoid"][(n + d) % 4])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,d,f", [(5000, 64, 40), (3000, 192, 100), (1024, 512, 512)])
def test_rows_that_are_alike(n, d, f, dtype):
    """The same row many times, and one gradient for all: what is lost of one term is lost of every one"""
    import torch
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, getattr(torch, dtype))
    _compare((bar[:1] / 8).expand(n, f), ((x[:1] / 8).expand(n, d), wg, wv, bg, bv), "silu")
