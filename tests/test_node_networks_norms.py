"""What the binding refuses of the norms' parameters that it takes for node networks, decided before any HIP call (no GPU needed)."""
import pytest

from paper_2506_02023_amd import binding as B


def _x():
    import torch
    return torch.zeros(5, 8), torch.ones(8)


@pytest.mark.parametrize("norm", ["post", "pre"])
@pytest.mark.parametrize("wrong", [lambda w: (w,), lambda w: (), lambda w: (w, None, None), lambda w: w, lambda w: [w], lambda w: 1.0])
def test_norms_are_pairs(norm, wrong):
    """One element less would move the next norm's parameters to another place"""
    x, w = _x()
    for call in (lambda k: B.mlip_residual(x, x, **k), lambda k: B.mlip_residual_grad(x, None, x, x, **k)):
        for other in (None, (w, w)):
            with pytest.raises(B.MlipError, match="pair"):
                call({norm: wrong(w), {"post": "pre", "pre": "post"}[norm]: other})
