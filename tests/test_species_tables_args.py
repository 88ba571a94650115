"""What the table and clipping calls refuse, decided before any HIP call (no GPU needed)."""
import ctypes

import pytest

from paper_2506_02023_amd import binding as B

EINVAL = -1
OK = 256      # an address that is never read: every call here is refused, or has nothing to do


def _embed(**k):
    a = dict(table=OK, table_dtype=0, n_rows=4, width=8, rs=8, cs=1, ids=OK, id_bits=32, n=5, scale=1.0, out=OK, out_dtype=0, os=8)
    a.update(k)
    return B.lib().mlip_embed(a["table"], a["table_dtype"], a["n_rows"], a["width"], a["rs"], a["cs"], a["ids"], a["id_bits"], a["n"],
                              a["scale"], a["out"], a["out_dtype"], a["os"], None)


def _grad(**k):
    a = dict(grad=OK, dtype=0, rs=8, cs=1, ids=OK, id_bits=32, n=5, n_rows=4, width=8, scale=1.0, acc=0, out=OK, out_dtype=0, os=8, ws=OK,
             ws_bytes=1 << 40)
    a.update(k)
    return B.lib().mlip_embed_grad(a["grad"], a["dtype"], a["rs"], a["cs"], a["ids"], a["id_bits"], a["n"], a["n_rows"], a["width"],
                                   a["scale"], a["acc"], a["out"], a["out_dtype"], a["os"], a["ws"], a["ws_bytes"], None)


COMMON = [dict(n=-1), dict(n=1 << 31), dict(n_rows=0), dict(n_rows=1 << 31), dict(width=0), dict(width=1 << 31), dict(ids=None),
          dict(id_bits=16), dict(ids=OK + 2), dict(ids=OK + 4, id_bits=64), dict(out=None), dict(out=OK + 2), dict(out=OK + 1, out_dtype=1),
          dict(out_dtype=3), dict(out_dtype=-1), dict(rs=-1), dict(cs=-1), dict(os=7), dict(rs=1 << 60), dict(cs=1 << 60), dict(os=1 << 60)]


@pytest.mark.parametrize("wrong", COMMON + [dict(table=None), dict(table=OK + 2), dict(table_dtype=7)])
def test_lookup_refuses(wrong):
    assert _embed(**wrong) == EINVAL
    assert B.lib().mlip_last_error()


@pytest.mark.parametrize("wrong", COMMON + [dict(grad=None), dict(grad=OK + 1, dtype=2), dict(dtype=7)])
def test_gradient_refuses(wrong):
    assert _grad(**wrong) == EINVAL
    assert B.lib().mlip_last_error()


def test_gradient_refuses_a_small_workspace():
    L = B.lib()
    for n, rows, width in ((5, 4, 8), (1_000_000, 8, 64), (100_000, 50_000, 8)):
        need = L.mlip_embed_grad_workspace(n, rows, width)
        if need:
            for wrong in (dict(ws=None), dict(ws=OK + 8), dict(ws_bytes=need - 1)):
                assert _grad(n=n, n_rows=rows, width=width, rs=width, os=width, **wrong) == EINVAL
            assert b"workspace" in L.mlip_last_error()
    assert L.mlip_embed_grad_workspace(-1, 4, 8) == 0


def test_workspace_of_sizes_that_are_refused():
    L = B.lib()
    for sizes in ((-1, 4, 8), (1 << 31, 4, 8), (5, 0, 8), (5, 1 << 31, 8), (5, 4, 0), (5, 4, (1 << 20) + 1), (5, 4, 1 << 62), (1 << 62, 1 << 62, 1 << 62)):
        assert L.mlip_embed_grad_workspace(*sizes) == 0
    assert L.mlip_embed_grad_workspace((1 << 31) - 1, (1 << 31) - 1, 1 << 20) > 0
    assert L.mlip_grad_workspace(-5) > 0


def test_lookup_of_nothing_is_no_error():
    assert _embed(n=0, ids=None, out=None) == 0


def _list(*tensors):
    return (B._Tensor * len(tensors))(*tensors), len(tensors)


@pytest.mark.parametrize("tensor", [(None, OK, 4, 0), (OK, OK, -1, 0), (OK, OK, (1 << 40) + 1, 0), (OK, OK, 4, 3), (OK + 2, OK, 4, 0),
                                    (OK + 1, OK, 4, 1)])
def test_norm_and_clip_refuse_a_tensor(tensor):
    L = B.lib()
    a, count = _list((OK, OK, 0, 0), tensor)
    assert L.mlip_grad_norm(a, count, OK, OK, 1 << 30, None) == EINVAL
    assert b"tensor 1" in L.mlip_last_error()
    assert L.mlip_clip_grads(a, count, 1.0, OK, OK, 1 << 30, None) == EINVAL


def test_norm_and_clip_refuse():
    L = B.lib()
    a, count = _list((OK, OK, 4, 0))
    ws = 1 << 30
    assert L.mlip_grad_norm(a, -1, OK, OK, ws, None) == EINVAL
    assert L.mlip_grad_norm(None, 1, OK, OK, ws, None) == EINVAL
    assert L.mlip_grad_norm(a, count, None, OK, ws, None) == EINVAL
    assert L.mlip_grad_norm(a, count, OK + 2, OK, ws, None) == EINVAL
    assert L.mlip_grad_norm(a, count, OK, None, ws, None) == EINVAL
    assert L.mlip_grad_norm(a, count, OK, OK, L.mlip_grad_workspace(count) - 1, None) == EINVAL
    for max_norm in (-1.0, float("nan")):
        assert L.mlip_clip_grads(a, count, max_norm, OK, OK, ws, None) == EINVAL
    for dst in (None, OK + 2):
        a, count = _list((OK, dst, 4, 0))
        assert L.mlip_clip_grads(a, count, 1.0, OK, OK, ws, None) == EINVAL


def test_dense_layouts():
    import torch
    t = torch.zeros(2, 3, 4)
    assert B._dense(t) and B._dense(t.permute(2, 0, 1)) and B._dense(torch.zeros(5, 1).t()) and B._dense(torch.zeros(()))
    assert not B._dense(t[:, :2]) and not B._dense(torch.zeros(1).expand(4)) and not B._dense(t[..., ::2])


def test_struct_of_the_binding_matches_the_header():
    assert ctypes.sizeof(B._Tensor) == 32 and B._Tensor.n.offset == 16 and B._Tensor.dtype.offset == 24


def test_binding_refuses():
    """Checks that the binding makes of tensors before it calls (CPU tensors are refused last, by their device)."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the device check needs no GPU only where there is none")
    t, s = torch.zeros(4, 8), torch.zeros(5, dtype=torch.int32)
    wrong = [lambda: B.mlip_embed(t.double(), s), lambda: B.mlip_embed(t[None], s), lambda: B.mlip_embed(t, s.short()),
             lambda: B.mlip_embed(t, s[:, None]), lambda: B.mlip_embed(t, torch.zeros(10, dtype=torch.int32)[::2]),
             lambda: B.mlip_embed(t, s, out=torch.zeros(5, 7)), lambda: B.mlip_embed(t, s, out=torch.zeros(8, 5).t()),
             lambda: B.mlip_embed_grad(torch.zeros(4, 8), s, 4), lambda: B.mlip_embed_grad(torch.zeros(5, 8), s, 4, accumulate=True),
             lambda: B.mlip_embed_grad(torch.zeros(5, 8), s, 4, out=torch.zeros(3, 8)),
             lambda: B.mlip_grad_norm([torch.zeros(3, dtype=torch.int32)]), lambda: B.mlip_grad_norm([torch.zeros(4, 4)[:, :2]]),
             lambda: B.mlip_clip_grads([t], 1.0, out=[]), lambda: B.mlip_clip_grads([t], 1.0, out=[torch.zeros(8, 4).t()])]
    for call in wrong:
        with pytest.raises(B.MlipError):
            call()
