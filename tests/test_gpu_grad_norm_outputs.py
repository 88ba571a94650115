"""The norm does not use its tensors' `dst`: whatever it holds, the call is the same one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 32768, 32768 - 8, 100_000])
def test_norm_whatever_the_outputs(n):
    """32768 fp32 elements from a whole line on are four tiles, which one block sums without scratch memory; counted from a place inside a line they would
    be five.  Norm and scratch memory are the same bits whatever address, of nothing, stands in `dst`."""
    import torch
    from paper_2506_02023_amd import binding as B
    L = B.lib()
    x = torch.as_tensor(np.random.default_rng(n).normal(size=n), dtype=torch.float32, device="cuda")
    assert x.data_ptr() % 128 == 0
    norm = torch.empty((), device="cuda")
    need = L.mlip_grad_workspace(1)
    seen = []
    for dst in (None, x.data_ptr(), 4, 1, 127, 2 ** 40 + 60):
        ws = torch.full((need,), 0xab, dtype=torch.uint8, device="cuda")
        a = (B._Tensor * 1)((x.data_ptr(), dst, n, 0))
        assert L.mlip_grad_norm(a, 1, norm.data_ptr(), ws.data_ptr(), need, B._stream()) == 0
        want = float(x.double().square().sum().sqrt())
        assert abs(float(norm) - want) <= (2.0 ** -24 + 2.0 ** -30) * want
        seen.append((norm.clone(), ws))
    for norm_k, ws_k in seen[1:]:
        assert torch.equal(norm_k, seen[0][0]) and torch.equal(ws_k, seen[0][1])
