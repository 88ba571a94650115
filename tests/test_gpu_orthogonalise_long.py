"""Orthogonal updates of few very long rows, whose sums have up to 2^20 terms, against the same iteration in 64 bits, to the tolerances of test_gpu_orthogonalise.py,
which do not grow with the length."""
import pytest

from test_gpu_orthogonalise import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 5000), (9000, 1), (2, 100_000), (33, 70_000), (1, 1 << 20), (130, 200_000), (40_000, 140), (5, 4096), (5, 4097), (3, 12_289)])
@pytest.mark.parametrize("kind", ["ones", "noise", "two sizes"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_long_rows(shape, kind, dtype):
    import torch
    import paper_2506_02023_amd as M
    g = torch.Generator(device="cuda").manual_seed(shape[0])
    m = torch.randn(shape, generator=g, device="cuda")
    if kind == "ones":
        m = torch.ones(shape, device="cuda")
    elif kind == "two sizes":       # a few large elements at the front of rows of equal ones
        m = torch.full(shape, 0.7, device="cuda") * m.sign()
        m[:3, :3] *= 100.0
    m = m.to(getattr(torch, dtype))
    _check(M.mlip_orthogonalise([m.clone()])[0], m, kind)
