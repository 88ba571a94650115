"""What the binding makes of lists of gradients, before the library is called (no GPU needed)."""
import pytest

from paper_2506_02023_amd import binding as B


@pytest.fixture
def cpu_tensors_pass(monkeypatch):
    """The device of CPU tensors, -1, taken for the current GPU, so that the lists can be looked at where there is none."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)


def _words(listed):
    held, address, count = listed
    assert address == held.buffer_info()[0]
    return held.tolist(), count


def test_any_iterable_of_gradients(cpu_tensors_pass):
    """Generators, iterators and tuples are what lists of the same tensors are, as gradients and as outputs."""
    import torch
    ts = [torch.zeros(5), torch.zeros((2, 3), dtype=torch.bfloat16), torch.zeros(0), torch.zeros((3, 4)).t()]
    out = [torch.empty_like(t) for t in ts]
    want, want_out = _words(B._tensor_list(ts, None)), _words(B._tensor_list(ts, out))
    assert want[1] == want_out[1] == 4 and want[0][2::4] == [5, 6, 0, 12] and want_out[0][1::4] == [t.data_ptr() for t in out]
    for make in (tuple, iter, lambda x: (t for t in x), lambda x: dict(enumerate(x)).values()):
        assert _words(B._tensor_list(make(ts), None)) == want
        assert _words(B._tensor_list(make(ts), make(out))) == want_out
    for wrong in (out[:3], out[:3] + [out[0]]):
        with pytest.raises(B.MlipError):
            B._tensor_list((t for t in ts), (t for t in wrong))
    assert _words(B._tensor_list(iter(()), None)) == ([], 0)
