"""Orthogonal updates of matrices of few directions and few different values, whose roundings do not average out, against the same iteration in 64 bits.

Tolerances are those of test_gpu_orthogonalise.py, and for bf16 and fp16 matrices its first part: before the result's own rounding a step is off by 2^-18 of
the matrix's norm, stretched by the steps behind it."""
import numpy as np
import pytest

from test_gpu_orthogonalise import _reference

pytestmark = pytest.mark.gpu

KINDS = ["rank1", "rank1 and noise", "rank2", "two rows", "ones", "signs", "two values"]


def _make(m, n, kind, dtype, seed=0):
    import torch
    rng = np.random.default_rng([m, n, seed])
    r = rng.normal
    if kind.startswith("rank"):
        k = int(kind[4])
        g = r(size=(m, k)) @ r(size=(k, n)) + ("noise" in kind) * 1e-3 * r(size=(m, n))
    elif kind == "two rows":
        g, row = 1e-3 * r(size=(m, n)), r(size=n)
        g[3], g[m - 5] = row, row + 0.01 * r(size=n)
    elif kind == "ones":
        g = np.ones((m, n))
    elif kind == "signs":
        g = 0.7 * np.sign(r(size=(m, 1))) * np.sign(r(size=(1, n)))
    else:
        g = np.where(np.arange(n) % 3 == 0, 0.3, 0.7) * np.sign(r(size=(m, 1)))
    return torch.as_tensor(g, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m,n", [(40, 60), (130, 130), (200, 300), (300, 130), (512, 512), (600, 2000), (1024, 1024)])
def test_structured(m, n, kind, dtype):
    """The result's own rounding: half a step for every element, and one of 2^-11 (fp32 sums and 22 bits) beside it that only counts where elements are small"""
    import torch
    import paper_2506_02023_amd as M
    g = _make(m, n, kind, getattr(torch, dtype))
    got = M.mlip_orthogonalise([g.clone()])[0]
    want, tol = _reference(g)
    u = torch.finfo(g.dtype).eps / 2
    off = float((got.double() - want).norm())
    assert off <= tol * (1 + u) + u * float(want.norm()) * 1.001 + 1e-30, f"off by {off / float(want.norm()):.2e}, tolerance {(tol + u * float(want.norm())) / float(want.norm()):.2e}"
    # a result that is right to fp32 before its rounding is one of the two neighbours of the exact value: most elements are the exact value's own rounding
    if dtype != "float32":
        own = want.to(g.dtype).double()
        assert float((got.double() - own).norm()) <= 0.25 * u * float(want.norm()) + 2 * tol
