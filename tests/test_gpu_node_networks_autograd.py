"""The gradient calls and the forward calls for node networks inside autograd, where they cannot do what is asked of them: an error, never a result that has lost its graph."""
import pytest

pytestmark = pytest.mark.gpu


def _inputs(n=20, d=16, f=12):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)

    def t(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    return dict(x=t(n, d), z=t(n, d), grad=t(n, f), dy=t(n, d), dn=t(n, d), wg=t(d, f), wv=t(d, f), b=t(f), w=t(d), w2=t(d), gate=t(n, 1), scale=t(d))


def _gradient_calls():
    import paper_2506_02023_amd as M
    return {"mlip_gated_grad": (lambda v: M.mlip_gated_grad(v["grad"], v["x"], v["wg"], v["wv"], v["b"]), ["grad", "x", "wg", "wv", "b"]),
            "mlip_residual_grad": (lambda v: M.mlip_residual_grad(v["dy"], v["dn"], v["x"], v["z"], v["gate"], v["scale"], (v["w"], None), (v["w2"], None)),
                                   ["dy", "dn", "x", "z", "gate", "scale", "w", "w2"]),
            "mlip_norm_grad": (lambda v: M.mlip_norm_grad(v["dn"], v["x"], v["w"]), ["dn", "x", "w"])}


def _flat(out):
    import torch
    return [] if out is None else [out] if torch.is_tensor(out) else [t for o in out for t in _flat(o)]


@pytest.mark.parametrize("name", ["mlip_gated_grad", "mlip_residual_grad", "mlip_norm_grad"])
def test_results_of_gradient_calls_stay_in_the_graph(name):
    """They need a gradient where an input does, are the same bits, and asking for the gradient raises"""
    import torch
    call, keys = _gradient_calls()[name]
    values = _inputs()
    want = _flat(call(values))
    assert not any(t.requires_grad for t in want)
    for key in keys:
        here = {**values, key: values[key].clone().requires_grad_()}
        got = _flat(call(here))
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)
        assert all(t.requires_grad for t in got), key
        with pytest.raises(RuntimeError, match=name):
            got[0].sum().backward()
        with torch.no_grad():
            assert not any(t.requires_grad for t in _flat(call(here)))


def test_forward_mode_is_refused():
    """A dual tensor's tangent is not lost in silence"""
    import torch
    import torch.autograd.forward_ad as fwd
    import paper_2506_02023_amd as M
    v = _inputs()
    calls = [lambda x: M.mlip_gated(x, v["wg"], v["wv"]), lambda x: M.mlip_residual(x, v["z"]), lambda x: M.mlip_norm(x), lambda x: M.mlip_gated_grad(v["grad"], x, v["wg"], v["wv"]),
             lambda x: M.mlip_residual_grad(v["dy"], None, x, v["z"]), lambda x: M.mlip_norm_grad(v["dn"], x)]
    plain = [_flat(c(v["x"])) for c in calls]
    with fwd.dual_level():
        dual = fwd.make_dual(v["x"], torch.ones_like(v["x"]))
        for call, want in zip(calls, plain):
            with pytest.raises((RuntimeError, NotImplementedError)):
                call(dual)
            assert all(torch.equal(a, b) for a, b in zip(_flat(call(v["x"])), want))       # (others' calls go on)
