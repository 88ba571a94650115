"""The arrays that the gradient of gated projections makes: one for each result, in the order of its weights, whatever their strides."""
import pytest

from test_gpu_gated import _make

pytestmark = pytest.mark.gpu


def test_each_result_is_made_once():
    import torch
    import paper_2506_02023_amd as M
    bar, inputs = _make(3000, 64, 32, torch.float32)
    M.mlip_gated_grad(bar, *inputs)
    made = torch.cuda.memory_stats()["allocation.all.allocated"]
    held = M.mlip_gated_grad(bar, *inputs)
    assert len(held) == 5 and torch.cuda.memory_stats()["allocation.all.allocated"] - made == 5 + 1     # and the scratch memory


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_orders_of_the_weights(dtype):
    """Transposed, cut out, every second row and column, broadcast: results as of copies, without gaps"""
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    n, d, f = 90, 40, 24
    bar, (x, wg, wv, bg, bv) = _make(n, d, f, dt)
    big = torch.zeros(2 * d, 3 * f, dtype=dt, device="cuda")
    big[::2, 1::3] = wg
    flat = torch.zeros(f, d + 5, dtype=dt, device="cuda")
    flat[:, :d] = wg.t()
    for w in (wg.t().contiguous().t(), big[::2, 1::3], flat[:, :d].t(), wg[:1].expand(d, f), wg[:, :1].expand(d, f)):
        want = M.mlip_gated_grad(bar, x, w.contiguous(), wv, bg, bv)
        got = M.mlip_gated_grad(bar, x, w, wv, bg, bv)
        for a, b in zip(got, want):
            assert a.shape == b.shape and torch.equal(a, b) and a.untyped_storage().nbytes() <= a.numel() * a.element_size()
        leaf = w.clone().requires_grad_() if w.stride() != wg.stride() else w.detach().requires_grad_()
        M.mlip_gated(x, leaf, wv, bg, bv).backward(bar)
        assert torch.equal(leaf.grad, want[1])
