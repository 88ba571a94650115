"""What the calls for node networks refuse, decided before any HIP call (no GPU needed)."""
import ctypes

import pytest

from paper_2506_02023_amd import binding as B

EINVAL = -1
OK = 256      # an address that is never read: every call here is refused, or has nothing to do
BIG = 1 << 50


def _gated(**k):
    a = dict(dtype=0, act=0, n=5, d=8, f=6, x=OK, x_rs=8, x_cs=1, wg=OK, wg_rs=6, wg_cs=1, wv=OK, wv_rs=6, wv_cs=1, bg=OK, bv=None)
    return B._Gated(**{**a, **k})


GATED = [dict(dtype=3), dict(dtype=-1), dict(act=4), dict(act=-1), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=65537), dict(f=0), dict(f=65537), dict(x=None), dict(wg=None),
         dict(wv=None), dict(x=OK + 2), dict(x=OK + 1, dtype=1), dict(wg=OK + 2), dict(bg=OK + 2), dict(bv=OK + 1), dict(x_rs=-1), dict(x_cs=-1), dict(wg_rs=-1), dict(wv_cs=-1),
         dict(x_rs=1 << 60), dict(wv_cs=1 << 60)]


@pytest.mark.parametrize("wrong", GATED)
def test_gated_refuses(wrong):
    L = B.lib()
    assert L.mlip_gated(_gated(**wrong), OK, 6, OK, BIG, None) == EINVAL and L.mlip_last_error()
    assert L.mlip_gated_grad(_gated(**wrong), B._GatedGrad(grad=OK, grad_rs=6, grad_cs=1), OK, BIG, None) == EINVAL
    assert L.mlip_gated_workspace(_gated(**wrong), 0) == L.mlip_gated_workspace(_gated(**wrong), 1) == 0


def test_gated_refuses_outputs_and_scratch():
    L = B.lib()
    need = L.mlip_gated_workspace(_gated(), 0)
    assert need > 0
    for out, rs, ws, size in ((None, 6, OK, BIG), (OK + 2, 6, OK, BIG), (OK, 5, OK, BIG), (OK, -1, OK, BIG), (OK, 6, None, BIG), (OK, 6, OK + 8, BIG), (OK, 6, OK, need - 1)):
        assert L.mlip_gated(_gated(), out, rs, ws, size, None) == EINVAL
    assert L.mlip_gated(None, OK, 6, OK, BIG, None) == EINVAL and L.mlip_gated_workspace(None, 0) == 0
    assert L.mlip_gated(_gated(n=0, x=None), None, 6, OK, BIG, None) == 0


@pytest.mark.parametrize("wrong", [dict(grad=None), dict(grad=OK + 2), dict(grad_rs=-1), dict(grad_cs=1 << 60), dict(x=OK + 2), dict(x_rs=7), dict(x_rs=-8), dict(wg=OK + 1), dict(wg_rs=5),
                                   dict(wv_rs=0), dict(wv_cs=0), dict(wv_rs=1, wv_cs=7), dict(bg=OK + 2), dict(bv=OK + 1)])
def test_gated_gradient_refuses(wrong):
    L = B.lib()
    a = dict(grad=OK, grad_rs=6, grad_cs=1, x=OK, x_rs=8, wg=OK, wg_rs=6, wg_cs=1, wv=OK, wv_rs=6, wv_cs=1, bg=OK, bv=OK)
    assert L.mlip_gated_grad(_gated(), B._GatedGrad(**{**a, **wrong}), OK, BIG, None) == EINVAL


def test_gated_gradient_refuses_scratch():
    L = B.lib()
    need = L.mlip_gated_workspace(_gated(), 1)
    for ws, size in ((None, BIG), (OK + 8, BIG), (OK, need - 1)):
        assert L.mlip_gated_grad(_gated(), B._GatedGrad(grad=OK, grad_rs=6, grad_cs=1), ws, size, None) == EINVAL
        assert b"workspace" in L.mlip_last_error()
    assert L.mlip_gated_grad(_gated(), None, OK, BIG, None) == EINVAL


def test_gated_workspace_of_the_largest_sizes():
    L = B.lib()
    k = dict(n=(1 << 31) - 1, d=65536, f=65536, x_rs=65536, wg_rs=65536, wv_rs=65536)
    assert 0 < L.mlip_gated_workspace(_gated(**k), 0) < L.mlip_gated_workspace(_gated(**k), 1)
    assert 0 < L.mlip_gated_workspace(_gated(n=(1 << 31) - 1, d=1, f=1), 1)
    for n in (0, 1):
        assert L.mlip_gated_workspace(_gated(n=n), 1) > 0


def _residual(**k):
    a = dict(dtype=1, param_dtype=0, kind=0, gate_kind=1, post=1, pre=1, n=5, width=8, eps=1e-6, factor=1.0, x=OK, x_rs=8, x_cs=1, z=OK, z_rs=8, z_cs=1, gate=OK, gate_rs=8, gate_cs=1,
             scale=OK, post_w=OK, post_b=OK, pre_w=OK, pre_b=OK)
    return B._Residual(**{**a, **k})


RESIDUAL = [dict(dtype=3), dict(dtype=-1), dict(param_dtype=2), dict(param_dtype=5), dict(kind=2), dict(kind=-1), dict(gate_kind=4), dict(gate_kind=-1), dict(n=-1), dict(n=1 << 31), dict(width=0),
            dict(width=8193), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(x=OK + 1), dict(x_rs=-1), dict(x_cs=1 << 60), dict(z=OK + 1), dict(z_cs=-1), dict(gate=None), dict(gate=OK + 1),
            dict(gate=None, gate_kind=2), dict(gate=None, gate_kind=3), dict(gate_rs=-1), dict(gate_rs=-1, gate_kind=2), dict(scale=OK + 2), dict(post_w=OK + 2), dict(post_b=OK + 2), dict(pre_w=OK + 2),
            dict(pre_b=OK + 2), dict(post=0), dict(pre=0), dict(z=None), dict(z=None, gate_kind=0, scale=None, post=0), dict(z=None, gate_kind=0, post=0, post_w=None, post_b=None)]


@pytest.mark.parametrize("wrong", RESIDUAL)
def test_residual_refuses(wrong):
    L = B.lib()
    assert L.mlip_residual(_residual(**wrong), OK, 8, OK, 8, None) == EINVAL and L.mlip_last_error()
    assert L.mlip_residual_grad(_residual(**wrong), B._ResidualGrad(y=OK, y_rs=8, y_cs=1), OK, BIG, None) == EINVAL


def test_residual_refuses_outputs():
    L = B.lib()
    alone = dict(z=None, gate_kind=0, scale=None, post=0, post_w=None, post_b=None)
    nothing = dict(pre=0, pre_w=None, pre_b=None)
    for call, y, y_rs, norm, n_rs in ((_residual(), OK + 1, 8, OK, 8), (_residual(), OK, 7, OK, 8), (_residual(), OK, 8, None, 8), (_residual(), OK, 8, OK, 7), (_residual(), OK, 8, OK + 1, 8),
                                      (_residual(**alone), OK, 8, OK, 8), (_residual(**nothing), OK, 8, OK, 8), (_residual(**nothing), None, 8, None, 8),
                                      (_residual(**alone, **nothing), None, 8, None, 8)):
        assert L.mlip_residual(call, y, y_rs, norm, n_rs, None) == EINVAL
    assert L.mlip_residual(None, OK, 8, OK, 8, None) == EINVAL
    assert L.mlip_residual(_residual(n=0, x=None, gate=None), None, 8, None, 8, None) == 0


@pytest.mark.parametrize("wrong", [dict(y=None, norm=None), dict(y=OK + 1), dict(y_rs=-1), dict(norm=OK + 1), dict(norm_cs=1 << 60), dict(x=OK + 1), dict(x_rs=7), dict(z=OK + 1), dict(z_rs=0),
                                   dict(gate=OK + 1), dict(gate_rs=7), dict(scale=OK + 2), dict(post_w=OK + 1), dict(post_b=OK + 2), dict(pre_w=OK + 2), dict(pre_b=OK + 2)])
def test_residual_gradient_refuses(wrong):
    L = B.lib()
    a = dict(y=OK, y_rs=8, y_cs=1, norm=OK, norm_rs=8, norm_cs=1, x=OK, x_rs=8, z=OK, z_rs=8, gate=OK, gate_rs=8, scale=OK, post_w=OK, post_b=OK, pre_w=OK, pre_b=OK)
    assert L.mlip_residual_grad(_residual(), B._ResidualGrad(**{**a, **wrong}), OK, BIG, None) == EINVAL


def test_residual_gradient_refuses_what_the_call_does_not_have():
    L = B.lib()
    for k, out in ((dict(gate_kind=0), dict(gate=OK, gate_rs=8)), (dict(scale=None), dict(scale=OK)), (dict(post_w=None), dict(post_w=OK)), (dict(post_b=None), dict(post_b=OK)),
                   (dict(pre_w=None), dict(pre_w=OK)), (dict(pre_b=None), dict(pre_b=OK)), (dict(pre=0, pre_w=None, pre_b=None), dict(norm=OK, norm_rs=8, norm_cs=1)),
                   (dict(gate_kind=2), dict(gate=OK, gate_rs=0))):
        assert L.mlip_residual_grad(_residual(**k), B._ResidualGrad(y=OK, y_rs=8, y_cs=1, **out), OK, BIG, None) == EINVAL
    n, width = 100_000, 64
    need = L.mlip_residual_grad_workspace(n, width)
    assert need > 0
    call = _residual(n=n, width=width, x_rs=64, z_rs=64, gate_rs=64)
    for ws, size in ((None, BIG), (OK + 8, BIG), (OK, need - 1)):
        assert L.mlip_residual_grad(call, B._ResidualGrad(y=OK, y_rs=64, y_cs=1, scale=OK), ws, size, None) == EINVAL
    assert L.mlip_residual_grad(_residual(), None, OK, BIG, None) == EINVAL
    assert L.mlip_residual_grad_workspace(-1, 64) == L.mlip_residual_grad_workspace(5, 0) == L.mlip_residual_grad_workspace(5, 8193) == 0
    assert L.mlip_residual_grad_workspace((1 << 31) - 1, 8192) > 0


def _matrix(**k):
    a = dict(src=OK, dst=OK, rows=4, cols=6, src_rs=6, src_cs=1, dst_rs=6, dst_cs=1, dtype=0)
    return B._Matrix(**{**a, **k})


@pytest.mark.parametrize("wrong", [dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 20) + 1), dict(cols=(1 << 20) + 1), dict(rows=32769, cols=32769),
                                   dict(rows=32768, cols=65536), dict(src=None), dict(dst=None), dict(src=OK + 2), dict(dst=OK + 1, dtype=1), dict(src_rs=-1), dict(src_cs=1 << 60), dict(dst_rs=5),
                                   dict(dst_cs=0), dict(dst_rs=1, dst_cs=3)])
def test_orthogonalise_refuses_a_matrix(wrong):
    L = B.lib()
    a = (B._Matrix * 2)(_matrix(), _matrix(**wrong))
    coef = (ctypes.c_double * 3)(1.5, -0.5, 0.0)
    assert L.mlip_orthogonalise(a, 2, 5, coef, 1e-7, 1.0, OK, BIG, None) == EINVAL
    assert b"matrix 1" in L.mlip_last_error()
    assert L.mlip_orthogonalise_workspace(a, 2) == 0


def test_orthogonalise_refuses():
    L = B.lib()
    a, coef = (B._Matrix * 1)(_matrix()), (ctypes.c_double * 3)(1.5, -0.5, 0.0)
    need = L.mlip_orthogonalise_workspace(a, 1)
    assert need > 0
    for args in ((a, -1, 5, coef, 1e-7, OK, BIG), (None, 1, 5, coef, 1e-7, OK, BIG), (a, 1, -1, coef, 1e-7, OK, BIG), (a, 1, 1001, coef, 1e-7, OK, BIG), (a, 1, 5, None, 1e-7, OK, BIG),
                 (a, 1, 5, coef, -1.0, OK, BIG), (a, 1, 5, coef, float("nan"), OK, BIG), (a, 1, 5, coef, 1e-7, None, BIG), (a, 1, 5, coef, 1e-7, OK + 8, BIG), (a, 1, 5, coef, 1e-7, OK, need - 1)):
        list_, count, steps, c, eps, ws, size = args
        assert L.mlip_orthogonalise(list_, count, steps, c, eps, 1.0, ws, size, None) == EINVAL
    assert L.mlip_orthogonalise(None, 0, 5, coef, 1e-7, 1.0, OK, BIG, None) == 0


def test_structs_of_the_binding_match_the_header():
    assert [ctypes.sizeof(s) for s in (B._Gated, B._GatedGrad, B._Residual, B._ResidualGrad, B._Matrix)] == [120, 104, 160, 136, 72]
    assert B._Residual.x.offset == 48 and B._Gated.bv.offset == 112 and B._Matrix.dtype.offset == 64


def test_binding_refuses():
    """Checks that the binding makes of tensors before it calls"""
    import torch
    x, w, b, v = torch.zeros(5, 8), torch.zeros(8, 6), torch.zeros(6), torch.zeros(8)
    half = x.bfloat16()
    wrong = [lambda: B.mlip_gated(x.double(), w, w), lambda: B.mlip_gated(x[0], w, w), lambda: B.mlip_gated(x, w.bfloat16(), w), lambda: B.mlip_gated(x, w, w[:, :5]), lambda: B.mlip_gated(x, w[:7], w[:7]),
             lambda: B.mlip_gated(x, w, w, b[:5]), lambda: B.mlip_gated(x, w, w, b, torch.zeros(12)[::2]), lambda: B.mlip_gated(x, w, w, act="tanh"), lambda: B.mlip_gated(x, b, w),
             lambda: B.mlip_gated_grad(torch.zeros(5, 5), x, w, w), lambda: B.mlip_gated_grad(torch.zeros(5, 6).half(), x, w, w),
             lambda: B.mlip_residual(x, x[:4]), lambda: B.mlip_residual(x, None), lambda: B.mlip_residual(x, half), lambda: B.mlip_residual(x, x, torch.zeros(5, 2)), lambda: B.mlip_residual(x, x, v.bfloat16()),
             lambda: B.mlip_residual(x, x, scale=v[:7]), lambda: B.mlip_residual(x, x, scale=v.half()), lambda: B.mlip_residual(half, half, scale=v.half()), lambda: B.mlip_residual(half, half, scale=v, post=(v.bfloat16(), None)),
             lambda: B.mlip_residual(x, x, kind="batch"), lambda: B.mlip_residual_grad(None, None, x, None), lambda: B.mlip_residual_grad(torch.zeros(4, 8), None, x, x), lambda: B.mlip_norm(x[0]), lambda: B.mlip_norm(x, v[:3]),
             lambda: B.mlip_norm_grad(half, x), lambda: B.mlip_orthogonalise([v]), lambda: B.mlip_orthogonalise([x], out=[]), lambda: B.mlip_orthogonalise([x], out=[torch.zeros(8, 5)]),
             lambda: B.mlip_orthogonalise([x.double()])]
    for call in wrong:
        with pytest.raises(B.MlipError):
            call()
