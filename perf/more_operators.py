"""The measured operators of training a potential's node networks: gated projections, norms around a block, orthogonal updates.

A block of a deep potential takes the atoms' (or edges') features x through a norm, a pair of gated projections and a projection
back, and adds the result to x under a gate; its weight matrices are trained with orthogonalised updates.  Per step of a fit:

  gated           h = phi(x Wg + bg, x Wv + bv) for every element, phi(g, v) = silu(g) v, gelu(g) v, sigmoid(g) v or sigmoid(g) silu(v),
  gated_grad      from dh: dx, dWg, dWv, dbg, dbv,
  residual        y = x + scale * gate * post(z), n = pre(y), with norms post and pre of the rows: (t - mean) / sqrt(mean of (t - mean)^2 + eps)
                  ("layer") or t / sqrt(mean of t^2 + eps) ("rms"), times weights and plus biases of the columns,
  residual_grad   from dy and dn: the gradients of x, z, gate, scale and of the norms' weights and biases,
  orthogonalise   X_0 = G / |G|, X_k+1 = a X_k + b (X_k X_k^T) X_k + c (X_k X_k^T)^2 X_k for each matrix of a list (its transpose where it has more
                  rows than columns), five steps.

exact() is the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ["silu", "gelu", "sigmoid", "silu_sigmoid"]
COEF = (3.4445, -4.7750, 2.0315)
STEPS = 5
MOST_FLOPS = 1.64e12     # of a drawn case
MOST = 134_000_000       # elements of one matrix of a drawn case


def _gated(op, n, d, f, dtype="f32", act="silu", bias=False, turned=False, gap=0, name=None):
    """n rows of d features into f.  turned: the weights lie as [f][d]; gap: elements between the rows of x and of dh."""
    c = dict(op=op, n=n, d=d, f=f, dtype=dtype, act=act, bias=bias, turned=turned, gap=gap)
    if name:
        c["name"] = name
    return c


def _residual(op, n, width, dtype="f32", params="f32", kind="rms", gate="none", scale=False, post=True, pre=True, bias=False, gap=0, name=None):
    """gate: "none", "full" [n, width], "row" [n, 1] or "col" [width]; gap: elements between the rows of the inputs; bias: of the norms."""
    c = dict(op=op, n=n, width=width, dtype=dtype, params=params, kind=kind, gate=gate, scale=scale, post=post, pre=pre, bias=bias, gap=gap)
    if name:
        c["name"] = name
    return c


def _ortho(shapes, dtype="f32", name=None):
    """shapes: "AxB*K" joined by "+": K matrices of A rows and B columns each"""
    c = dict(op="orthogonalise", shapes=shapes, dtype=dtype)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one small structure of 108 atoms: latency is all there is
        _gated("gated", 108, 64, 128, name="gated_108"),
        # the million-atom system's node update, both sides activated, with biases
        _gated("gated", 1_000_188, 64, 128, "bf16", "silu_sigmoid", bias=True, name="gated_1m"),
        # wide features of a large batch in fp32, an odd hidden width, rows cut out of a wider matrix
        _gated("gated", 32_768, 512, 1365, "f32", "gelu", bias=True, turned=True, gap=3, name="gated_wide_f32"),
        # a step of a fit on a few structures
        _gated("gated_grad", 500, 64, 256, "f32", bias=True, name="gated_grad_500"),
        # the 202,612-atom system in fp32, an odd hidden width
        _gated("gated_grad", 202_612, 128, 341, "f32", bias=True, name="gated_grad_200k"),
        # wide features of a large batch
        _gated("gated_grad", 32_768, 1024, 4096, "bf16", turned=True, name="gated_grad_wide"),
        # the million-atom system: sum, both norms and a gate for every atom in one go
        _residual("residual", 1_000_188, 64, "bf16", kind="layer", gate="row", scale=True, bias=True, name="residual_1m"),
        # a small structure
        _residual("residual_grad", 108, 64, "f32", scale=True, name="residual_grad_108"),
        # the million-atom system with a gate for every element, weights in fp32
        _residual("residual_grad", 1_000_188, 128, "bf16", kind="layer", gate="full", scale=True, bias=True, name="residual_grad_1m"),
        # wide rows of an odd width in fp32, cut out of wider matrices
        _residual("residual_grad", 32_771, 1365, "f32", kind="rms", gate="col", gap=3, name="residual_grad_wide"),
        # the gradients of one model of the smaller sizes
        _ortho("64x64*9+64x128*6+8x64*3", "f32", name="ortho_model"),
        # the gradients of wide blocks, some with more rows than columns
        _ortho("1024x4096*8+4096x1024*4", "bf16", name="ortho_large"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high))))) if high > low else int(low)


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_grad", "gated_grad", "gated_grad", "residual", "residual", "residual_grad", "residual_grad",
                     "residual_grad", "orthogonalise", "orthogonalise", "orthogonalise"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("gated", "gated_grad"):
        d = rng.choice([32, 64, 64, 128, 256, _log(rng, 1, 1024), _log(rng, 16, 1024)])
        f = min(4096, rng.choice([2 * d, 4 * d, 8 * d // 3, _log(rng, 1, 4096), _log(rng, 16, 4096)]))
        f = max(1, f)
        return _gated(op, _log(rng, 1, min(1_000_188, MOST / max(d, f), MOST_FLOPS / (12 * d * f))), d, f, dtype, rng.choice(ACTS),
                      rng.random() < 0.5, rng.random() < 0.5, rng.choice([0, 0, 1, 3, 8]))
    if op == "orthogonalise":
        shapes, cost = [], 0
        for _ in range(rng.choice([1, 1, 2, 3])):
            a, b, k = _log(rng, 1, 4096), _log(rng, 1, 4096), _log(rng, 1, 24)
            m, most = min(a, b), max(a, b)
            one = STEPS * (4.0 * m * m * most + 2.0 * m ** 3)
            k = max(1, min(k, int((MOST_FLOPS * 0.7 - cost) / one)))
            if cost + k * one > MOST_FLOPS * 0.7:
                a, b, k, one = 64, 128, 3, 0
            cost += k * one
            shapes.append(f"{a}x{b}*{k}")
        return _ortho("+".join(shapes), dtype)
    width = rng.choice([32, 64, 64, 128, _log(rng, 8, 8192), _log(rng, 8, 8192), _log(rng, 256, 8192)])
    return _residual(op, _log(rng, 1, min(1_000_188, MOST / width)), width, dtype, rng.choice(["f32", dtype]), rng.choice(["rms", "layer"]),
                     rng.choice(["none", "full", "row", "col"]), rng.random() < 0.5, rng.random() < 0.8, rng.random() < 0.8, rng.random() < 0.5,
                     rng.choice([0, 0, 1, 3, 8]))


# ---------------------------------------------------------------- inputs

def _matrix(rows, width, gap, dtype, g, std=1.0, mean=0.0):
    m = torch.randn((rows, width + gap), generator=g, device="cuda").mul_(std).add_(mean)
    return m.to(DTYPES[dtype])[:, :width]


def _vector(width, dtype, g, mean, std):
    return torch.randn(width, generator=g, device="cuda").mul_(std).add_(mean).to(DTYPES[dtype])


def _shapes(case):
    return [tuple(map(int, s.split("*")[0].split("x"))) for s in case["shapes"].split("+") for _ in range(int(s.split("*")[1]))]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "orthogonalise":
        # a gradient: products of a batch's features that share a few directions, and what differs from atom to atom
        st["matrices"] = []
        for a, b in _shapes(case):
            r = max(1, min(a, b) // 8)
            m = torch.randn((a, r), generator=g, device="cuda") @ torch.randn((r, b), generator=g, device="cuda") / math.sqrt(r)
            st["matrices"].append((m + 0.3 * torch.randn((a, b), generator=g, device="cuda")).mul_(1e-3).to(DTYPES[case["dtype"]]))
        st["out"] = [torch.empty_like(m) for m in st["matrices"]]
        return st
    if case["op"] in ("gated", "gated_grad"):
        n, d, f, dt = case["n"], case["d"], case["f"], case["dtype"]
        st["x"] = _matrix(n, d, case["gap"], dt, g)
        for w in ("wg", "wv"):
            m = _matrix(f if case["turned"] else d, d if case["turned"] else f, 0, dt, g, 1.0 / math.sqrt(d))
            st[w] = m.t() if case["turned"] else m
        st["bg"], st["bv"] = (_vector(f, dt, g, 0.0, 0.2) if case["bias"] else None for _ in range(2))
        if case["op"] == "gated_grad":
            st["dh"] = _matrix(n, f, case["gap"], dt, g, 0.1)
        return st
    n, width, dt, gap = case["n"], case["width"], case["dtype"], case["gap"]
    st["x"] = _matrix(n, width, gap, dt, g, 1.5)
    st["z"] = _matrix(n, width, gap, dt, g, 0.7, 0.2)
    st["gate"] = None
    if case["gate"] != "none":
        shape = {"full": (n, width), "row": (n, 1), "col": (1, width)}[case["gate"]]
        gate = torch.sigmoid(torch.randn(shape, generator=g, device="cuda")).to(DTYPES[dt])
        st["gate"] = gate[0] if case["gate"] == "col" else gate
    st["scale"] = _vector(width, case["params"], g, 0.3, 0.1) if case["scale"] else None
    for norm in ("post", "pre"):
        st[norm] = None
        if case[norm]:
            st[norm] = (_vector(width, case["params"], g, 1.0, 0.2), _vector(width, case["params"], g, 0.0, 0.2) if case["bias"] else None)
    if case["op"] == "residual_grad":
        st["dy"] = _matrix(n, width, gap, dt, g, 0.1)
        st["dn"] = _matrix(n, width, gap, dt, g, 0.1) if case["pre"] else None
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    return _run_own(c, state) if own else _run_plain(c, state)


def _flat(outputs):
    """The tensors of nested tuples, those that are None left out"""
    if outputs is None or torch.is_tensor(outputs):
        return [] if outputs is None else [outputs]
    return [t for o in outputs for t in _flat(o)]


def _run_own(c, s):
    import paper_2506_02023_amd as M
    if c["op"] == "gated":
        return M.mlip_gated(s["x"], s["wg"], s["wv"], s["bg"], s["bv"], act=c["act"])
    if c["op"] == "gated_grad":
        return _flat(M.mlip_gated_grad(s["dh"], s["x"], s["wg"], s["wv"], s["bg"], s["bv"], act=c["act"]))
    if c["op"] == "residual":
        return _flat(M.mlip_residual(s["x"], s["z"], s["gate"], s["scale"], post=s["post"], pre=s["pre"], kind=c["kind"], eps=1e-6))
    if c["op"] == "residual_grad":
        return _flat(M.mlip_residual_grad(s["dy"], s["dn"], s["x"], s["z"], s["gate"], s["scale"], post=s["post"], pre=s["pre"], kind=c["kind"], eps=1e-6))
    M.mlip_orthogonalise(s["matrices"], steps=STEPS, coefficients=COEF, out=s["out"])
    return s["out"]


def _phi(act, g, v):
    """(phi, d phi / d g, d phi / d v)"""
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * c * v, (c + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))) * v, g * c
    s = torch.sigmoid(g)
    if act == "silu":
        return g * s * v, s * (1 + g * (1 - s)) * v, g * s
    if act == "sigmoid":
        return s * v, s * (1 - s) * v, s
    t = torch.sigmoid(v)
    return s * v * t, s * (1 - s) * v * t, s * t * (1 + v * (1 - t))


def _norm(kind, t):
    """(normalised rows, 1 / their deviation)"""
    if kind == "layer":
        t = t - t.mean(1, keepdim=True)
    r = torch.rsqrt(t.square().mean(1, keepdim=True) + 1e-6)
    return t * r, r


def _norm_back(kind, bar, hat, r):
    d = bar - hat * (bar * hat).mean(1, keepdim=True)
    if kind == "layer":
        d = d - bar.mean(1, keepdim=True)
    return d * r


def _run_plain(c, s):
    if c["op"] == "orthogonalise":
        return [_ortho_plain(m) for m in s["matrices"]]
    f32 = {k: v.float() for k, v in s.items() if torch.is_tensor(v)}
    dt = DTYPES[c["dtype"]]
    if c["op"] in ("gated", "gated_grad"):
        x, wg, wv = f32["x"], f32["wg"], f32["wv"]
        g, v = x @ wg, x @ wv
        if c["bias"]:
            g, v = g + f32["bg"], v + f32["bv"]
        h, hg, hv = _phi(c["act"], g, v)
        if c["op"] == "gated":
            return h.to(dt)
        dg, dv = f32["dh"] * hg, f32["dh"] * hv
        grads = [dg @ wg.t() + dv @ wv.t(), x.t() @ dg, x.t() @ dv] + ([dg.sum(0), dv.sum(0)] if c["bias"] else [])
        return [t.to(dt) for t in grads]
    pdt = DTYPES[c["params"]]
    zh, zr = _norm(c["kind"], f32["z"]) if c["post"] else (f32["z"], None)
    p = zh
    if c["post"]:
        p = zh * s["post"][0].float() + (s["post"][1].float() if c["bias"] else 0.0)
    gate, scale = f32.get("gate"), f32.get("scale")
    t = (1.0 if gate is None else gate) * (1.0 if scale is None else scale)
    y = f32["x"] + t * p
    yh, yr = _norm(c["kind"], y) if c["pre"] else (None, None)
    if c["op"] == "residual":
        return [y.to(dt)] + ([(yh * s["pre"][0].float() + (s["pre"][1].float() if c["bias"] else 0.0)).to(dt)] if c["pre"] else [])
    dy, dpre = f32["dy"], []
    if c["pre"]:
        dn = f32["dn"]
        dpre = [(dn * yh).sum(0).to(pdt)] + ([dn.sum(0).to(pdt)] if c["bias"] else [])
        dy = dy + _norm_back(c["kind"], dn * s["pre"][0].float(), yh, yr)
    dp, dt_ = dy * t, dy * p
    dz, dpost = dp, []
    if c["post"]:
        dpost = [(dp * zh).sum(0).to(pdt)] + ([dp.sum(0).to(pdt)] if c["bias"] else [])
        dz = _norm_back(c["kind"], dp * s["post"][0].float(), zh, zr)
    out = [dy.to(dt), dz.to(dt)]
    if gate is not None:
        dgate = dt_ if scale is None else dt_ * scale
        out.append((dgate if c["gate"] == "full" else dgate.sum(1, keepdim=True) if c["gate"] == "row" else dgate.sum(0)).to(dt))
    if scale is not None:
        out.append((dt_ if gate is None else dt_ * gate).sum(0).to(pdt))
    return out + dpost + dpre


def _ortho_plain(m):
    x = m.float()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = (x / x.double().square().sum().sqrt().clamp(min=1e-7)).float()
    a, b, c = COEF
    for _ in range(STEPS):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return (x.t() if tall else x).to(m.dtype).contiguous()


def work(case):
    if case["op"] == "orthogonalise":
        shapes = [(min(s), max(s)) for s in _shapes(case)]
        # X X^T and its square are symmetric: half of each
        return {"bytes": sum(2 * m * n for m, n in shapes) * SIZE[case["dtype"]], "flops": sum(STEPS * (3.0 * m * m * n + m ** 3) for m, n in shapes)}
    size = SIZE[case["dtype"]]
    if case["op"] in ("gated", "gated_grad"):
        n, d, f = case["n"], case["d"], case["f"]
        weights = 2 * d * f + (2 * f if case["bias"] else 0)
        if case["op"] == "gated":
            return {"bytes": (n * (d + f) + weights) * size, "flops": 4.0 * n * d * f}
        return {"bytes": (n * (2 * d + f) + 2 * weights) * size, "flops": 12.0 * n * d * f}
    n, width = case["n"], case["width"]
    gate = {"none": 0, "full": n * width, "row": n, "col": width}[case["gate"]]
    params = (case["scale"] + (case["post"] + case["pre"]) * (2 if case["bias"] else 1)) * width * SIZE[case["params"]]
    if case["op"] == "residual":
        return {"bytes": ((3 + case["pre"]) * n * width + gate) * size + params, "flops": 15.0 * n * width}
    return {"bytes": ((5 + case["pre"]) * n * width + 2 * gate) * size + 2 * params, "flops": 40.0 * n * width}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _leaf(t):
    return None if t is None else t.double().detach().requires_grad_()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalise":
        return [_ortho_exact(m.double()) for m in s["matrices"]]
    with torch.enable_grad():
        if case["op"] in ("gated", "gated_grad"):
            names = ["x", "wg", "wv", "bg", "bv"]
            leaves = [_leaf(s[k]) for k in names]
            x, wg, wv, bg, bv = leaves
            g, v = (torch.mm(x, w) if b is None else torch.addmm(b, x, w) for w, b in ((wg, bg), (wv, bv)))
            if case["act"] == "gelu":
                h = g * torch.special.ndtr(g) * v
            else:
                gated = 1 / (1 + torch.exp(-g))
                h = gated * (g * v if case["act"] == "silu" else v if case["act"] == "sigmoid" else v / (1 + torch.exp(-v)))
            if case["op"] == "gated":
                return h.detach()
            return list(torch.autograd.grad(h, [t for t in leaves if t is not None], s["dh"].double()))
        x, z, gate, scale = (_leaf(s[k]) for k in ("x", "z", "gate", "scale"))
        post, pre = ([_leaf(t) for t in s[k]] if s[k] else [] for k in ("post", "pre"))

        def norm(t, params):
            if case["kind"] == "layer":
                var, mean = torch.var_mean(t, dim=1, keepdim=True, correction=0)
                t = (t - mean) / torch.sqrt(var + 1e-6)
            else:
                t = t / torch.sqrt(torch.linalg.vecdot(t, t)[:, None] / t.shape[1] + 1e-6)
            t = t * params[0]
            return t if params[1] is None else t + params[1]

        inner = norm(z, post) if post else z
        for factor in (gate, scale):
            inner = inner if factor is None else inner * factor
        y = x + inner
        outs = [y] + ([norm(y, pre)] if pre else [])
        if case["op"] == "residual":
            return [t.detach() for t in outs]
        leaves = [t for t in [x, z, gate, scale, *post, *pre] if t is not None]
        return list(torch.autograd.grad(outs, leaves, [s["dy"].double()] + ([s["dn"].double()] if pre else [])))


def _ortho_exact(g):
    """All steps on the matrix of the rows' products alone, with the polynomials' product applied at the end"""
    if g.shape[0] > g.shape[1]:
        return _ortho_exact(g.t()).t().contiguous()
    x = g / max(float(torch.linalg.vector_norm(g)), 1e-7)
    a, b, c = COEF
    gram, total = x.mm(x.t()), torch.eye(g.shape[0], dtype=torch.float64, device=g.device)
    for _ in range(STEPS):
        step = b * gram + c * gram.mm(gram)
        step.diagonal().add_(a)
        total, gram = step.mm(total), step.mm(gram).mm(step)
    return total.mm(x)
