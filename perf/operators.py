"""The measured operators of fitting a potential's per-species parameters: table lookup, its gradient, the gradients' norm.

A potential keeps one row of parameters for each chemical species (the embedding the message passing starts from, reference
energies and scales of the atoms' energies) or for each pair of species.  Fitting them takes, at every step,

  lookup   out[i, :] = scale * table[id_i, :], a row of zeros where id_i < 0 (places that pad a batch of structures),
  grad     dtable[s, :] = scale * sum over i with id_i = s of dout[i, :], rows that no atom has are zero,
  norm     n = sqrt(sum over all gradient tensors and their elements of x^2),
  clip     out = x * c with c = max_norm / n if n > max_norm is finite, c = 1 otherwise, for every element; and n.

exact() is the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MOST = 131072 * 1024     # elements of the rows of one lookup or gradient
MOST_CLIP = 1 << 28      # elements of the tensors of one clip


def _table(op, n, rows, width, dtype="f32", out="f32", ids="i32", spread="uniform", pad=0.0, gap=0, scale=1.0, name=None):
    """n ids into a table of rows x width.  spread: how often a row comes up, "uniform", "zipf" (the k-th most frequent one 1/k as often)
    or "runs" (uniform, the ids in runs as in a file of structures sorted by element); pad: share of ids that are -1; gap: elements
    between the end of a row of the input matrix (lookup: table, grad: incoming gradient) and the start of the next."""
    c = dict(op=op, n=n, rows=rows, width=width, dtype=dtype, out=out, ids=ids, spread=spread, pad=pad, gap=gap, scale=scale)
    if name:
        c["name"] = name
    return c


def _list(op, tensors, total, kinds="f32", shape="mixed", max_norm=1.0, name=None):
    """Gradients of `tensors` tensors with about `total` elements together.  shape: "mixed" (sizes spread over their logarithm) or "even";
    kinds: the types, one after the other, joined by "+"."""
    c = dict(op=op, tensors=tensors, total=total, kinds=kinds, shape=shape, max_norm=max_norm)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one small structure of 108 atoms, four species, the narrow model's embedding: latency is all there is
        _table("lookup", 108, 4, 32, name="lookup_108"),
        # the million-atom system's embedding
        _table("lookup", 1_000_188, 8, 64, name="lookup_1m"),
        # a padded batch of structures in bf16, all elements of the periodic table, an odd width, rows cut out of a wider table
        _table("lookup", 202_612, 119, 77, "bf16", "bf16", spread="zipf", pad=0.1, gap=5, scale=8.775, name="lookup_ragged_bf16"),
        # a wide table of many rows (environment types), 64-bit ids as torch makes them, the result in bf16
        _table("lookup", 131_072, 50_021, 1024, "f32", "bf16", ids="i64", spread="zipf", scale=32.0, name="lookup_large_table"),
        # the gradients of the same: the smallest step of a fit
        _table("grad", 108, 4, 32, name="grad_108"),
        # the million-atom system: very few rows, so that every row sums over 125,000 atoms
        _table("grad", 1_000_188, 8, 64, name="grad_1m"),
        # scale and shift of the atoms' energies by element, a million atoms in runs of the same element
        _table("grad", 1_000_188, 89, 2, spread="runs", name="grad_shift_1m"),
        # pairs of species, an odd width, bf16 gradients summed into fp32, padded, rows cut out of a wider matrix
        _table("grad", 300_007, 14_161, 33, "bf16", "f32", spread="zipf", pad=0.1, gap=7, scale=0.125, name="grad_pairs_bf16"),
        # a wide table of many rows, most of which no atom of the batch has
        _table("grad", 131_072, 50_021, 1024, "bf16", "f32", ids="i64", spread="zipf", scale=32.0, name="grad_large_table"),
        # the gradients of one model of this size: seven small tensors
        _list("clip", 7, 60_000, name="clip_model"),
        # several hundred tensors of very different sizes, two types in one list; only their norm, as a run's log has it
        _list("norm", 400, 60_000_000, "bf16+f32", max_norm=0.0, name="norm_400"),
        # the largest: a gigabyte of gradients in two hundred tensors
        _list("clip", 200, 250_000_000, "f32", name="clip_large"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup", "lookup", "grad", "grad", "grad", "grad", "clip", "clip", "norm"])
    if op in ("clip", "norm"):
        kinds = rng.choice(["f32", "bf16", "f16+f32", "bf16+f32"])
        tensors = max(_log(rng, 1, 500), kinds.count("+") + 1)
        return _list(op, tensors, max(tensors, _log(rng, 1000, MOST_CLIP * 0.9)), kinds, rng.choice(["mixed", "even"]),
                     max_norm=0.0 if op == "norm" else round(math.exp(rng.uniform(-2, 2)), 4))
    width = rng.choice([1, 2, 3, 16, 32, 64, 64, 128, _log(rng, 1, 1024), _log(rng, 1, 1024)])
    n = _log(rng, 1, min(2_000_000, MOST * 0.9 // width))
    rows = rng.choice([1, 4, 8, 89, 119, _log(rng, 1, 50_000), _log(rng, 1, 50_000)])
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    return _table(op, n, rows, width, dtype, rng.choice([dtype, "f32"]), rng.choice(["i32", "i32", "i64"]),
                  rng.choice(["uniform", "zipf", "runs"]), rng.choice([0.0, 0.0, 0.1, 0.5]), rng.choice([0, 0, 0, 1, 4, 5]),
                  rng.choice([1.0, 0.125, round(math.sqrt(width), 3)]))


# ---------------------------------------------------------------- inputs

def _ids(case, g):
    n, rows = case["n"], case["rows"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if case["spread"] == "runs":     # about 100 runs
        u = u[torch.arange(n, device="cuda") // max(1, n // 100)]
    if case["spread"] == "zipf":
        k = torch.exp(u * math.log(rows + 1)).long() - 1
        k = torch.randperm(rows, generator=g, device="cuda")[k.clamp(0, rows - 1)]
    else:
        k = (u * rows).long().clamp(max=rows - 1)
    k = torch.where(torch.rand(n, generator=g, device="cuda") < case["pad"], -1, k)
    return k.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _matrix(rows, width, gap, dtype, g, mean):
    m = torch.randn((rows, width + gap), generator=g, device="cuda").mul_(0.5).add_(mean)
    return m.to(DTYPES[dtype])[:, :width]


def _sizes(case):
    """Sizes of the list's tensors (a model's: they go with the case, not with the seed), of the case's total within rounding"""
    k, r = case["tensors"], torch.Generator().manual_seed(case["tensors"])
    w = torch.ones(k, dtype=torch.float64) if case["shape"] == "even" else torch.exp(torch.rand(k, generator=r, dtype=torch.float64) * math.log(1e4))
    return [max(1, int(x)) for x in (w / w.sum() * case["total"]).tolist()]


def _tensors(case, seed):
    """(tensors, the flat buffer of each type that they are views of): gradients lie in flat buffers, as where they are exchanged in buckets"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    kinds, sizes = case["kinds"].split("+"), _sizes(case)
    flat, views = {}, [None] * len(sizes)
    for i, kind in enumerate(kinds):
        mine = sizes[i::len(kinds)]
        flat[kind] = (torch.randn(sum(mine), generator=g, device="cuda") * (10.0 / math.sqrt(case["total"]))).to(DTYPES[kind])
        views[i::len(kinds)] = flat[kind].split(mine)
    return views, flat


def prepare(case, seed):
    if case["op"] in ("clip", "norm"):
        views, flat = _tensors(case, seed)
        st = dict(case=case, tensors=views)
        if case["op"] == "clip":
            st["flat"] = {k: torch.empty_like(f) for k, f in flat.items()}
            kinds = list(flat)
            st["out"] = [None] * len(views)
            for i, k in enumerate(kinds):
                st["out"][i::len(kinds)] = st["flat"][k].split([v.numel() for v in views[i::len(kinds)]])
        return st
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = _ids(case, g)
    rows = case["rows"] if case["op"] == "lookup" else case["n"]
    m = _matrix(rows, case["width"], case["gap"], case["dtype"], g, 0.0 if case["op"] == "lookup" else 0.1)
    return dict(case=case, ids=ids, m=m)


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    return _run_own(c, state) if own else _run_plain(c, state)


def _run_own(c, state):
    import paper_2506_02023_amd as M
    if c["op"] == "lookup":
        out = torch.empty((c["n"], c["width"]), dtype=DTYPES[c["out"]], device="cuda")
        return M.mlip_embed(state["m"], state["ids"], c["scale"], out=out)
    if c["op"] == "grad":
        out = torch.empty((c["rows"], c["width"]), dtype=DTYPES[c["out"]], device="cuda")
        return M.mlip_embed_grad(state["m"], state["ids"], c["rows"], c["scale"], out=out)
    if c["op"] == "norm":
        return M.mlip_grad_norm(state["tensors"])
    norm = M.mlip_clip_grads(state["tensors"], c["max_norm"], out=state["out"])
    return [norm, state["flat"]]


def _run_plain(c, state):
    if c["op"] in ("lookup", "grad"):
        ids, m = state["ids"].long(), state["m"].float()
        there = (ids >= 0)[:, None]
        if c["op"] == "lookup":
            return torch.where(there, m[ids.clamp(min=0)] * c["scale"], 0.0).to(DTYPES[c["out"]])
        parts = max(1, min(256, 65536 // c["rows"]))   # few rows: summed in parts, so that no sum runs over 100,000s of atoms in 32 bits
        sums = torch.zeros((parts * c["rows"], c["width"]), device="cuda")
        part = torch.arange(c["n"], device="cuda") * parts // c["n"] * c["rows"]
        sums.index_add_(0, ids.clamp(min=0) + part, torch.where(there, m, 0.0))
        return (sums.view(parts, c["rows"], c["width"]).sum(0) * c["scale"]).to(DTYPES[c["out"]])
    norm = torch.stack([t.float().square().sum() for t in state["tensors"]]).sum().sqrt()
    if c["op"] == "norm":
        return norm
    coef = torch.where((norm > c["max_norm"]) & torch.isfinite(norm), c["max_norm"] / norm, 1.0)
    kinds = list(state["flat"])
    return [norm, {k: torch.cat([(t.float() * coef).to(t.dtype) for t in state["tensors"][i::len(kinds)]]) for i, k in enumerate(kinds)}]


def work(case):
    if case["op"] in ("clip", "norm"):
        kinds, sizes = case["kinds"].split("+"), _sizes(case)
        moved = sum(sum(sizes[i::len(kinds)]) * SIZE[k] for i, k in enumerate(kinds))
        return {"bytes": moved * (2 if case["op"] == "clip" else 1), "flops": sum(sizes) * (3 if case["op"] == "clip" else 2)}
    n, rows, width, id_bytes = case["n"], case["rows"], case["width"], case["n"] * (4 if case["ids"] == "i32" else 8)
    real = n * (1 - case["pad"])
    if case["op"] == "lookup":   # no more rows of the table than there are ids
        return {"bytes": id_bytes + min(rows, real) * width * SIZE[case["dtype"]] + n * width * SIZE[case["out"]], "flops": real * width}
    return {"bytes": id_bytes + real * width * SIZE[case["dtype"]] + rows * width * SIZE[case["out"]], "flops": real * width}


# ---------------------------------------------------------------- from the definitions, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("clip", "norm"):
        square = 0.0
        for t in st["tensors"]:
            square += float(torch.linalg.vecdot(t.double(), t.double()))
        norm = math.sqrt(square)
        if case["op"] == "norm":
            return torch.tensor(norm, dtype=torch.float64)
        c = case["max_norm"] / norm if norm > case["max_norm"] else 1.0
        _, flat = _tensors(case, seed)
        return [torch.tensor(norm, dtype=torch.float64), {k: f.double() * c for k, f in flat.items()}]
    ids, m = st["ids"].long(), st["m"].double()
    if case["op"] == "lookup":
        padded = torch.cat([m, torch.zeros((1, case["width"]), dtype=torch.float64, device="cuda")])   # the id -1 is its last row
        return torch.index_select(padded, 0, torch.remainder(ids, case["rows"] + 1)) * case["scale"]
    # running sums of the rows in the order of their ids, and their differences at the ends of each id's rows
    ids, order = torch.sort(ids, stable=True)
    ends = torch.searchsorted(ids, torch.arange(-1, case["rows"], device="cuda"), right=True)
    parts = []
    for cols in m.split(128, dim=1):
        run_sum = torch.zeros((case["n"] + 1, cols.shape[1]), dtype=torch.float64, device="cuda")
        torch.cumsum(cols[order], 0, out=run_sum[1:])
        at = run_sum[ends]
        parts.append(at[1:] - at[:-1])
    return torch.cat(parts, dim=1) * case["scale"]
