"""Gates far from zero, where phi and its derivatives are small: relative to their own size, against 64-bit arithmetic.

x = [g, 1] and weights of zeros and ones make g any number of the type and v = 1 exactly, so that all that is off is phi.  exp(-|t|) is off by the roundings of
its argument, 2^-24 |t| each, and some of its own; the normal distribution's tail at g by those times g^2.  Counted: 2^-20 + 4 (g^2 + 2) 2^-24 of the
value for the gelu, 2^-20 + 4 (|g| + 2) 2^-24 for the others, of the sizes of what is added, and half a step of the type for each rounding to it."""
import pytest

pytestmark = pytest.mark.gpu

U24 = 2.0 ** -24


def _values(dtype, top):
    import torch
    return torch.cat([torch.linspace(-top, top, 2999, device="cuda"), torch.linspace(4, 9, 200, device="cuda"), -torch.linspace(4, 9, 200, device="cuda")]).to(dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("d", [2, 160])
@pytest.mark.parametrize("act,top", [("gelu", 12.0), ("sigmoid", 60.0), ("silu", 60.0), ("silu_sigmoid", 60.0)])
def test_tails(act, top, d, dtype):
    import torch
    import paper_2506_02023_amd as M
    dt = getattr(torch, dtype)
    t = _values(dt, top)
    x = torch.zeros(len(t), d, dtype=dt, device="cuda")
    x[:, 0], x[:, 1] = t, 1
    wg, wv = torch.zeros(d, 1, dtype=dt, device="cuda"), torch.zeros(d, 1, dtype=dt, device="cuda")
    wg[0], wv[1] = 1, 1
    got = M.mlip_gated(x, wg, wv, act=act)[:, 0].double()
    back = M.mlip_gated_grad(torch.ones(len(t), 1, dtype=dt, device="cuda"), x, wg, wv, act=act)[0].double()
    g = t.double()
    if act == "gelu":
        s, p = 0.5 * torch.erfc(g * -0.5 ** 0.5), torch.exp(-0.5 * g * g) * 0.3989422804014327
        h, hg, size_g, hv, size_v = g * s, s + g * p, s + g.abs() * p, g * s, (g * s).abs()
    else:
        s, q = torch.sigmoid(g), torch.sigmoid(-g)
        one, oneq = torch.sigmoid(torch.ones_like(g)), torch.sigmoid(-torch.ones_like(g))
        if act == "sigmoid":
            h, hg, hv = s, s * q, s
        elif act == "silu":
            h, hg, hv = g * s, s * (1 + g * q), g * s
        else:
            h, hg, hv = s * one, s * q * one, s * one * (1 + oneq)
        size_g, size_v = (s * (1 + g.abs() * q) if act == "silu" else hg.abs()), hv.abs()
    e = 2.0 ** -20 + 4 * ((g * g if act == "gelu" else g.abs()) + 2) * U24
    u = torch.finfo(dt).eps / 2
    least = torch.finfo(dt).smallest_normal * 2
    # (the gradients of g and v are rounded to the type before the product with weights of one, which is rounded again)
    for what, a, b, size, roundings in (("h", got, h, h.abs(), 1), ("dg", back[:, 0], hg, size_g, 2), ("dv", back[:, 1], hv, size_v, 2)):
        off = (a - b).abs() - (e * size + roundings * u * (1 + u) * (b.abs() + e * size) + least)
        k = int(off.argmax())
        assert float(off[k]) <= 0, f"{what} at {float(g[k])}: {float(a[k])} for {float(b[k])}"
