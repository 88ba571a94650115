"""Orthogonal updates without steps of matrices that are not finite, on all ways that a matrix may go."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 1), (40, 60), (200, 300), (300, 130)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_no_value_of_a_matrix_that_is_not_finite_is(shape, dtype, steps):
    import torch
    import paper_2506_02023_amd as M
    for bad in (float("inf"), -float("inf"), float("nan")):
        g = torch.ones(shape, dtype=getattr(torch, dtype), device="cuda")
        clean = g.clone()
        g[shape[0] // 2, shape[1] // 3] = bad
        out = M.mlip_orthogonalise([g, clean], steps=steps)
        assert not bool(out[0].isfinite().any()) and bool(out[1].isfinite().all())
