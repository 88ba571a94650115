"""Table lookup by species and its gradient against plain sums in 64 bits.

Bounds, from the roundings that the header names (u = 2^-24 is half a unit of the last place of fp32 relative to the value, u_out that of
the output's type): a looked-up value is one fp32 product rounded once more, so its error is at most (u + u_out (1 + u)) |value|; it equals torch's
fp32 product rounded to the type, bit for bit.  A gradient sums runs of at most 1024 atoms in fp32, each addition rounding by at most u of a partial
sum that is at most the sum of magnitudes, then runs in fp64: at most 1024 u sum|scale g| + (u + u_out)(1 + 1024 u) |value|, plus half the
smallest subnormal of the output's type.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
RUN = 1024


def _types():
    import torch
    return {"f32": (torch.float32, 0.0, 0.0), "bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


def _matrix(rng, rows, width, dtype, layout):
    """A matrix of a layout: "rows" one after another, "gap" between them (at an odd offset), "columns" one after another."""
    import torch
    dt = _types()[dtype][0]
    v = torch.as_tensor(rng.normal(0.1, 1.0, (rows, width)), dtype=torch.float32)
    if layout == "gap":
        m = torch.zeros(rows * (width + 3) + 1, dtype=dt, device="cuda")[1:].view(rows, width + 3)[:, :width]
    elif layout == "columns":
        m = torch.zeros((width, rows), dtype=dt, device="cuda").t()
    else:
        m = torch.zeros((rows, width), dtype=dt, device="cuda")
    m.copy_(v)
    return m


def _species(rng, n, rows, kind="uniform"):
    if kind == "one":
        return np.full(n, rows // 2)
    if kind == "runs":
        return np.sort(rng.integers(0, rows, n))
    if kind == "hot":       # half of the atoms have one species
        return np.where(rng.random(n) < 0.5, rows - 1, rng.integers(0, rows, n))
    if kind == "padded":
        return np.where(rng.random(n) < 0.3, -1 - rng.integers(0, 5, n), rng.integers(0, rows, n))
    return rng.integers(0, rows, n)


def _sums(g, ids, rows):
    """(sums, sums of magnitudes) by id in fp64"""
    ok = (ids >= 0) & (ids < rows)
    s, a = np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1]))
    order = np.argsort(ids[ok], kind="stable")
    k, v = ids[ok][order], g[ok][order]
    if len(k):
        start = np.flatnonzero(np.r_[True, k[1:] != k[:-1]])
        s[k[start]] = np.add.reduceat(v, start, axis=0)
        a[k[start]] = np.add.reduceat(np.abs(v), start, axis=0)
    return s, a


def _check_grad(g, species, rows, out_name, scale=1.0, layout_out=None):
    import torch
    import paper_2506_02023_amd as M
    dt, u_out, tiny = _types()[out_name]
    out = torch.full((rows, g.shape[1]), float("nan"), dtype=dt, device="cuda") if layout_out is None else layout_out
    M.mlip_embed_grad(g, species, rows, scale, out=out)
    s, a = _sums(g.double().cpu().numpy(), species.cpu().numpy().astype(np.int64), rows)
    s, a = s * scale, a * abs(scale)
    err = np.abs(out.double().cpu().numpy() - s)
    bound = RUN * U * a + (U + u_out) * (1 + RUN * U) * np.abs(s) + tiny
    assert (err <= bound).all(), (err - bound).max()
    return out


# widths that are a power of two, odd, one, more than a wavefront's lanes; rows from one to more than any fast path keeps at hand
SHAPES = [(1, 1, 1), (1, 8, 64), (2, 3, 5), (63, 4, 32), (64, 4, 32), (65, 4, 32), (108, 4, 32), (300, 1, 64), (500, 119, 1), (777, 89, 2),
          (1023, 8, 64), (1025, 8, 65), (2000, 119, 77), (4097, 160, 64), (4097, 161, 64), (5000, 700, 33), (3000, 5000, 16), (20000, 2, 64),
          (20011, 4, 3), (30000, 300, 130), (12345, 14161, 33), (9000, 50021, 8), (2500, 40, 1024), (70000, 3, 1), (40000, 1100, 256)]


@pytest.mark.parametrize("n,rows,width", SHAPES)
@pytest.mark.parametrize("kind", ["uniform", "hot", "padded"])
def test_gradient(n, rows, width, kind):
    import torch
    rng = np.random.default_rng([n, rows, width, len(kind)])
    g = _matrix(rng, n, width, "f32", "rows")
    species = torch.as_tensor(_species(rng, n, rows, kind), dtype=torch.int32, device="cuda")
    _check_grad(g, species, rows, "f32")


@pytest.mark.parametrize("layout", ["rows", "gap", "columns"])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,rows,width", [(700, 9, 30), (3001, 1234, 40), (40, 3, 200)])
def test_gradient_types_and_layouts(n, rows, width, dtype, out, layout):
    import torch
    rng = np.random.default_rng([n, rows, width])
    g = _matrix(rng, n, width, dtype, layout)
    species = torch.as_tensor(_species(rng, n, rows, "padded"), dtype=torch.int64, device="cuda")
    whole = torch.full((rows, width + 5), 7.0, dtype=_types()[out][0], device="cuda")
    _check_grad(g, species, rows, out, scale=0.25, layout_out=whole[:, 1:width + 1])
    assert (whole[:, 0] == 7).all() and (whole[:, width + 1:] == 7).all()     # nothing beside the output is written


@pytest.mark.parametrize("n,rows,width", [(50, 4, 8), (5000, 4, 8), (5000, 3000, 8), (100, 3000, 70)])
def test_gradient_long_runs_of_a_species(n, rows, width):
    import torch
    rng = np.random.default_rng([n, rows, width, 2])
    for kind in ("runs", "one"):
        species = torch.as_tensor(_species(rng, n, rows, kind), dtype=torch.int32, device="cuda")
        _check_grad(_matrix(rng, n, width, "f32", "rows"), species, rows, "f32")


@pytest.mark.parametrize("rows", [4, 5000])
def test_gradient_of_a_broadcast(rows):
    """The energy's own gradient is the same number for every atom: an expanded tensor."""
    import torch
    rng = np.random.default_rng(rows)
    n = 6000
    species = torch.as_tensor(_species(rng, n, rows), dtype=torch.int32, device="cuda")
    one = torch.tensor(0.75, device="cuda")
    out = _check_grad(one.expand(n, 3), species, rows, "f32")
    counts = np.bincount(species.cpu().numpy(), minlength=rows)
    assert np.array_equal(out.cpu().numpy(), np.repeat(0.75 * counts[:, None], 3, axis=1))      # whole multiples of 3/4: no rounding


@pytest.mark.parametrize("n,rows", [(0, 5), (0, 3000), (300, 6), (300, 4000), (9000, 6), (9000, 4000)])
def test_gradient_accumulates(n, rows):
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng([n, rows])
    g = _matrix(rng, n, 12, "f32", "rows")
    species = torch.as_tensor(_species(rng, n, rows), dtype=torch.int32, device="cuda")
    old = torch.as_tensor(rng.normal(size=(rows, 12)), dtype=torch.float32, device="cuda")
    out = old.clone()
    assert M.mlip_embed_grad(g, species, rows, 2.0, out=out, accumulate=True) is out
    s, a = _sums(g.double().cpu().numpy(), species.cpu().numpy().astype(np.int64), rows)
    s = 2 * s + old.double().cpu().numpy()
    assert (np.abs(out.double().cpu().numpy() - s) <= 2 * RUN * U * a + 2 * U * np.abs(s)).all()
    out = M.mlip_embed_grad(g, species, rows, 2.0)
    if n == 0:
        assert (out == 0).all()


@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("n,rows", [(200, 7), (5000, 7), (5000, 4000)])
def test_ids_without_a_row(n, rows, bits):
    """Negative ids and ids from n_rows on, with NaN and infinities in the gradients at their places: nothing of them comes in."""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng([n, rows, bits])
    dt = torch.int32 if bits == 32 else torch.int64
    ids = _species(rng, n, rows)
    out_ids = [-1, -2 ** 31, rows, rows + 1, 2 ** 31 - 1] + ([-2 ** 63, 2 ** 32, 2 ** 32 + 1, 2 ** 63 - 1] if bits == 64 else [])
    at = rng.choice(n, 100, replace=False)
    ids = ids.astype(np.int64)
    ids[at] = np.resize(out_ids, 100)
    g = rng.normal(size=(n, 16)).astype(np.float32)
    g[at[:50]], g[at[50:]] = np.nan, np.inf
    species = torch.as_tensor(ids, device="cuda").to(dt)
    s, a = _sums(g, ids, rows)
    out = M.mlip_embed_grad(torch.as_tensor(g, device="cuda"), species, rows)
    assert (np.abs(out.double().cpu().numpy() - s) <= RUN * U * a + 2 * U * np.abs(s)).all()
    table = torch.as_tensor(rng.normal(size=(rows, 16)), dtype=torch.float32, device="cuda")
    r = M.mlip_embed(table, species).cpu().numpy()
    ok = (ids >= 0) & (ids < rows)
    assert np.array_equal(r[ok], table.cpu().numpy()[ids[ok]]) and (r[ids < 0] == 0).all() and np.isnan(r[ids >= rows]).all()
    none = torch.full((n,), -1, dtype=dt, device="cuda")
    assert (M.mlip_embed_grad(torch.as_tensor(g, device="cuda"), none, rows) == 0).all()


@pytest.mark.parametrize("n,rows,width", [(100, 5, 8), (6000, 5, 8), (6000, 5, 70), (6000, 2000, 8)])
def test_values_that_are_not_finite_stay_with_their_species_and_column(n, rows, width):
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng([n, rows, width])
    ids = _species(rng, n, rows)
    ids[[3, 50, 51]] = [0, 1, 1]
    g = rng.normal(size=(n, width)).astype(np.float32)
    g[3, 1], g[50, 2], g[51, 2], g[50, 3] = np.nan, np.inf, -np.inf, np.inf
    out = M.mlip_embed_grad(torch.as_tensor(g, device="cuda"), torch.as_tensor(ids, dtype=torch.int32, device="cuda"), rows).cpu().numpy()
    bad = ~np.isfinite(out)
    assert bad.sum() == 3 and np.isnan(out[0, 1]) and np.isnan(out[1, 2]) and out[1, 3] == np.inf


@pytest.mark.parametrize("n,rows,width", [(5, 3, 4), (3000, 40, 6), (3000, 2000, 6)])
def test_gradient_is_the_lookups_derivative(n, rows, width):
    """Loss sum(w * lookup): its difference quotient for single table elements.  Table, step and scale are powers of two or small whole
    numbers, so the lookup's values are exact and the quotient is the sum of w up to the sum's own rounding."""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng([n, rows])
    table = torch.as_tensor(rng.integers(-8, 8, (rows, width)), dtype=torch.float32, device="cuda")
    species = torch.as_tensor(_species(rng, n, rows, "padded"), dtype=torch.int32, device="cuda")
    w = torch.as_tensor(rng.normal(size=(n, width)), dtype=torch.float32, device="cuda")
    grad = M.mlip_embed_grad(w, species, rows, 0.5).cpu().numpy()

    def loss(t):
        return float((w.double() * M.mlip_embed(t, species, 0.5).double()).sum())

    magnitude = float(w.double().abs().sum())
    for r, f in [(0, 0), (rows - 1, width - 1), *zip(rng.integers(0, rows, 6), rng.integers(0, width, 6))]:
        up, down = table.clone(), table.clone()
        up[r, f] += 1.0
        down[r, f] -= 1.0
        assert abs((loss(up) - loss(down)) / 2 - grad[r, f]) <= (RUN * U + 1e-12) * magnitude


@pytest.mark.parametrize("layout", ["rows", "gap", "columns"])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (1000, 5, 2), (108, 4, 32), (999, 17, 77), (70, 300, 1030), (2049, 8, 64)])
def test_lookup(n, rows, width, dtype, out, layout):
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng([n, rows, width])
    table = _matrix(rng, rows, width, dtype, layout)
    ids = _species(rng, n, rows, "padded")
    dt, u_out, tiny = _types()[out]
    for id_type, whole in ((torch.int32, torch.full((n, width + 3), 7.0, dtype=dt, device="cuda")), (torch.int64, None)):
        species = torch.as_tensor(ids, dtype=id_type, device="cuda")
        got = torch.empty((n, width), dtype=dt, device="cuda") if whole is None else whole[:, 1:width + 1]
        assert M.mlip_embed(table, species, 1.7, out=got) is got
        if whole is not None:
            assert (whole[:, 0] == 7).all() and (whole[:, width + 1:] == 7).all()
        scale = np.float32(1.7)
        want = torch.where((species >= 0)[:, None], table.float()[species.long().clamp(min=0)] * float(scale), 0.0).to(dt)
        assert torch.equal(got, want)
        exact = np.where(ids[:, None] >= 0, table.double().cpu().numpy()[np.maximum(ids, 0)] * float(scale), 0.0)
        assert (np.abs(got.double().cpu().numpy() - exact) <= (U + u_out * (1 + U)) * np.abs(exact) + tiny).all()


def test_vectors_and_defaults():
    """Tables of one number per species are vectors; outputs are made where none are given."""
    import torch
    import paper_2506_02023_amd as M
    shift = torch.tensor([1.0, -2.0, 4.0], dtype=torch.bfloat16, device="cuda")
    species = torch.tensor([2, 0, -1, 2, 1], device="cuda")
    rows = M.mlip_embed(shift, species, 0.5)
    assert rows.dtype == torch.bfloat16 and rows.tolist() == [2.0, 0.5, 0.0, 2.0, -1.0]
    assert M.mlip_embed_grad(rows, species, 4, 2.0).tolist() == [1.0, -2.0, 8.0, 0.0]
    assert M.mlip_embed(shift[::2], species.clamp(max=1)).tolist() == [4.0, 1.0, 0.0, 4.0, 4.0]
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert M.mlip_embed(shift, none).shape == (0,)
    assert M.mlip_embed(torch.ones((3, 7), device="cuda"), none).shape == (0, 7)


def test_same_bits_every_time():
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(5)
    for n, rows, width in ((100_003, 7, 64), (100_003, 119, 9), (60_001, 9000, 40), (3000, 2000, 40)):
        g = _matrix(rng, n, width, "f32", "rows")
        species = torch.as_tensor(_species(rng, n, rows, "hot"), dtype=torch.int32, device="cuda")
        first = M.mlip_embed_grad(g, species, rows)
        for _ in range(3):
            assert torch.equal(M.mlip_embed_grad(g, species, rows), first)


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^32 bytes and 2^31 elements: its last rows are read and written at their places."""
    import torch
    import paper_2506_02023_amd as M
    n, width = 17_000_000, 130
    species = (torch.arange(n, device="cuda") % 3).to(torch.int32)
    table = torch.tensor([[1.0], [2.0], [3.0]], dtype=torch.bfloat16, device="cuda").expand(3, width)
    rows = M.mlip_embed(table, species, out=torch.empty((n, width), dtype=torch.bfloat16, device="cuda"))
    assert n * width > 2 ** 31
    for i in (0, 1, n // 2, 2 ** 31 // width + 1, n - 2, n - 1):
        assert (rows[i] == i % 3 + 1).all()
    species[:] = -1
    species[-2:] = torch.tensor([1, 4000], dtype=torch.int32)
    for s, m in ((1, 3), (4000, 5000)):
        out = M.mlip_embed_grad(rows, species, m)
        assert (out[1] == (n - 2) % 3 + 1).all() and (out[2:4000] == 0).all()
        assert m < 4000 or (out[4000] == (n - 1) % 3 + 1).all()


def test_streams_and_graphs():
    """On a side stream, and captured and replayed with other work between the replays."""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(8)
    side = torch.cuda.Stream()
    for n, rows, width in ((300, 6, 32), (50_000, 6, 32), (50_000, 3000, 32), (2000, 3000, 32)):
        g = _matrix(rng, n, width, "f32", "rows")
        table = _matrix(rng, rows, width, "f32", "rows")
        species = torch.as_tensor(_species(rng, n, rows), dtype=torch.int32, device="cuda")
        want, want_rows = M.mlip_embed_grad(g, species, rows), M.mlip_embed(table, species, 3.0)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got, got_rows = M.mlip_embed_grad(g, species, rows), M.mlip_embed(table, species, 3.0)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want) and torch.equal(got_rows, want_rows)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            rows_out = M.mlip_embed(table, species, 3.0)
            grad_out = M.mlip_embed_grad(g, species, rows)
        for k in range(4):
            rows_out.fill_(-1)
            grad_out.fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(rows_out, want_rows) and torch.equal(grad_out, want), k
            g.mul_(2.0)
            table.mul_(2.0)
            want, want_rows = M.mlip_embed_grad(g, species, rows), M.mlip_embed(table, species, 3.0)


# around the sizes at which another way is taken: rows whose tables still fit the wavefronts' LDS, lists of one sort tile, a block's few steps
LIMITS = [(4097, 111, 64), (4097, 112, 64), (4097, 113, 64), (900, 160, 32), (5000, 161, 32), (6000, 254, 16), (6000, 255, 16), (6000, 256, 16),
          (2047, 300, 20), (2048, 300, 20), (2049, 300, 20), (4096, 2000, 5), (1024, 4, 64), (1025, 4, 64), (65535, 255, 2), (65537, 256, 2),
          (2100, 65535, 3), (2100, 65536, 3), (300, 70000, 4), (5000, 400, 512), (2500, 300, 257)]


@pytest.mark.parametrize("n,rows,width", LIMITS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_at_the_limits_of_the_ways(n, rows, width, dtype):
    import torch
    for kind in ("uniform", "hot"):
        rng = np.random.default_rng([n, rows, width, len(kind)])
        species = torch.as_tensor(_species(rng, n, rows, kind), dtype=torch.int32, device="cuda")
        _check_grad(_matrix(rng, n, width, dtype, "rows"), species, rows, dtype)
        _check_grad(_matrix(rng, n, width, dtype, "gap"), species, rows, "f32", scale=3.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_arrays_larger_than_the_caches(dtype):
    """Gradients and results beyond 100 MB are read and written past the caches"""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(4)
    width = 72 if dtype == "f32" else 520
    n = 110_000_000 // (width * (4 if dtype == "f32" else 2))
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn((n, width), generator=gen, device="cuda").to(_types()[dtype][0])
    for rows in (8, 9000):
        species = torch.as_tensor(_species(rng, n, rows, "hot"), dtype=torch.int32, device="cuda")
        out = M.mlip_embed_grad(g, species, rows, out=torch.empty((rows, width), device="cuda")).double()
        z = torch.zeros((rows, width), dtype=torch.float64, device="cuda")
        s, a = z.index_add(0, species.long(), g.double()), z.index_add(0, species.long(), g.double().abs())
        assert ((out - s).abs() <= RUN * U * a + 2 * U * s.abs()).all()
        table = g[:rows]
        assert torch.equal(M.mlip_embed(table, species), table[species.long()])
    del out, s, a, z


@pytest.mark.parametrize("rows", [5, 700])
def test_sums_of_subnormal_numbers(rows):
    """fp32 numbers below the normal range are not flushed: whole multiples of the smallest one add up exactly"""
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(rows)
    k = rng.integers(-50, 50, (3000, 8))
    species = rng.integers(0, rows, 3000)
    g = torch.as_tensor((k * 2.0 ** -149).astype(np.float32), device="cuda")
    out = M.mlip_embed_grad(g, torch.as_tensor(species, device="cuda"), rows).double().cpu().numpy()
    want = np.zeros((rows, 8))
    np.add.at(want, species, k)
    assert np.array_equal(out * 2.0 ** 149, want)


@pytest.mark.parametrize("n", [0, 700, 3000])
def test_a_table_of_many_more_rows_than_atoms(n):
    import torch
    import paper_2506_02023_amd as M
    rng = np.random.default_rng(n)
    rows = 3_000_000
    g = _matrix(rng, n, 5, "f32", "rows")
    ids = _species(rng, n, rows)
    out = torch.full((rows, 5), 9.0, device="cuda")
    M.mlip_embed_grad(g, torch.as_tensor(ids, dtype=torch.int64, device="cuda"), rows, out=out)
    s, a = _sums(g.double().cpu().numpy(), ids, rows)
    assert (np.abs(out.double().cpu().numpy() - s) <= RUN * U * a + 2 * U * np.abs(s)).all()


@pytest.mark.parametrize("width", [33, 59, 64, 90])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_results_of_any_alignment(width, dtype):
    """Results beyond 100 MB whose rows begin at any alignment, with and without gaps between them"""
    import torch
    import paper_2506_02023_amd as M
    dt = _types()[dtype][0]
    n = 104_000_000 // (width * (4 if dtype == "f32" else 2))
    gen = torch.Generator(device="cuda").manual_seed(width)
    table = torch.randn((300, width), generator=gen, device="cuda").to(dt)
    species = torch.randint(-3, 300, (n,), generator=gen, device="cuda")
    want = torch.where((species >= 0)[:, None], table[species.clamp(min=0)], 0.0)
    assert torch.equal(M.mlip_embed(table, species), want)
    for offset, gap in ((1, 0), (0, 3), (5, 7)):
        whole = torch.full((offset + n * (width + gap),), 7.0, dtype=dt, device="cuda")
        out = whole[offset:].view(n, width + gap)[:, :width]
        M.mlip_embed(table, species, out=out)
        assert torch.equal(out, want) and (whole[:offset] == 7).all() and (whole[offset:].view(n, width + gap)[:, width:] == 7).all()


@pytest.mark.parametrize("n,rows,width", [(5000, 80, 64), (5000, 81, 64), (4096, 144, 64), (4096, 145, 64), (5000, 128, 32), (5000, 129, 32), (5000, 224, 16),
                                          (5000, 225, 16), (30000, 8, 257), (30000, 8, 500), (40000, 60, 512), (2000, 3, 4200), (60, 5, 9000)])
def test_gradient_of_few_rows_and_tiles_of_columns(n, rows, width):
    import torch
    rng = np.random.default_rng([n, rows, width])
    species = torch.as_tensor(_species(rng, n, rows, "hot"), dtype=torch.int32, device="cuda")
    for dtype, layout in (("f32", "rows"), ("bf16", "rows"), ("f32", "gap")):
        _check_grad(_matrix(rng, n, width, dtype, layout), species, rows, "f32")
