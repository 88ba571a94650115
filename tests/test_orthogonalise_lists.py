"""What the binding refuses of the lists that it takes for orthogonal updates, decided before any HIP call (no GPU needed)."""
import pytest

from paper_2506_02023_amd import binding as B


def test_a_matrix_twice(monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)      # (get_device() of a CPU tensor)
    a, b = torch.ones(4, 4), torch.ones(4, 4)
    stack = torch.ones(3, 4, 4)
    for updates, out in (([a, a], None), ([a, b, a], None), ([stack, stack[1]], None), ([a, b], [b, a]), ([a, b], [b, torch.ones(4, 4)]), ([a, b], [torch.empty(4, 4)] * 2), ([a, a], [a, torch.empty(4, 4)]), ([a, a], [torch.empty(4, 4), a]),
                         ([stack], [torch.empty(1, 4, 4).expand(3, 4, 4)])):
        with pytest.raises(B.MlipError, match="matrix"):
            B.mlip_orthogonalise(updates, out=out)


def test_lists_that_are_taken(monkeypatch):
    """The same source twice, results in place beside others, empty matrices: reach the library"""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)

    class Reached(Exception):
        pass

    def library():
        raise Reached
    monkeypatch.setattr(B, "lib", library)
    a, b, none = torch.ones(4, 4), torch.ones(4, 4), torch.empty(0, 4)
    for updates, out in (([a, b], None), ([a, a], [torch.empty(4, 4), torch.empty(4, 4)]), ([a, b], [a, torch.empty(4, 4)]), ([none, none, a], None), ([none, a], [torch.empty(0, 4), a]),
                         ([torch.ones(3, 4, 4)], None)):
        with pytest.raises(Reached):
            B.mlip_orthogonalise(updates, out=out)
