"""The gradient of a residual sum whose norm nobody used: as of the sum without a norm, whatever the norm of such rows would be."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", [64, 77, 700])
def test_no_gradient_comes_through_an_unused_norm(width, kind):
    import torch
    import paper_2506_02023_amd as M
    g = torch.Generator(device="cuda").manual_seed(width)
    x, z, dy = (torch.randn(30, width, generator=g, device="cuda") for _ in range(3))
    scale, w = torch.rand(width, generator=g, device="cuda"), torch.rand(width, generator=g, device="cuda")
    x[3], z[3] = 0.0, 0.0                   # with eps = 0 this row's norm is NaN
    x[7, 5] = float("inf")
    x[8] = 3e38
    z[8] = 3e38
    args = dict(scale=scale, kind=kind, eps=0.0)
    want = M.mlip_residual_grad(dy, None, x, z, **args)
    got = M.mlip_residual_grad(dy, None, x, z, pre=(w, None), **args)
    for a, b in zip(got[:4], want[:4]):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    assert torch.equal(got[0], dy) and bool((got[5][0] == 0).all())
    leaves = [t.clone().requires_grad_() for t in (x, z)]
    y, _ = M.mlip_residual(*leaves, pre=(w, None), **args)
    y.backward(dy)
    assert torch.equal(leaves[0].grad, dy) and torch.equal(leaves[1].grad, want[1])
