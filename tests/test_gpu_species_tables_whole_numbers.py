"""Gradients of small odd whole numbers: every partial sum is a whole number below 2^24, exact in fp32 in whatever order, so the result is compared for equality and an
atom that is left out, counted twice or put into another row changes it by an odd number.  Results in bf16 and fp16 are those numbers rounded once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _odd(gen, shape, dtype):
    import torch
    return (torch.randint(-4, 4, shape, generator=gen, device="cuda", dtype=torch.int8) * 2 + 1).to(dtype)


def _ids(gen, n, rows, kind):
    """kind: "even" over all rows; "hot": half of the atoms in the last row, and some that pad or have no row"""
    import torch
    ids = torch.randint(0, rows, (n,), generator=gen, device="cuda")
    if kind == "hot":
        u = torch.rand(n, generator=gen, device="cuda")
        ids = torch.where(u < 0.5, rows - 1, torch.where(u < 0.55, -1, torch.where(u < 0.6, rows, ids)))
    return ids.to(torch.int32)


def _want(g, ids, rows, old=None, scale=1.0):
    """Differences of running sums over the atoms in the order of their ids, in fp64, where sums of whole numbers are exact"""
    import torch
    sorted_ids, order = torch.sort(ids, stable=True)
    ends = torch.searchsorted(sorted_ids, torch.arange(-1, rows, dtype=ids.dtype, device="cuda"), right=True)
    parts = []
    for cols in g.split(128, dim=1):
        sums = torch.zeros((len(ids) + 1, cols.shape[1]), dtype=torch.float64, device="cuda")
        torch.cumsum(cols[order].double(), 0, out=sums[1:])
        parts.append(sums[ends[1:]] - sums[ends[:-1]])
    s = torch.cat(parts, 1) * scale
    assert float(s.abs().max()) < 2 ** 24
    return s if old is None else s + old.double()


def _check(n, rows, width, dtype, kind, offset=0, gap=0, seed=0):
    import torch
    import paper_2506_02023_amd as M
    gen = torch.Generator(device="cuda").manual_seed(n * 31 + rows * 7 + width + seed)
    whole = _odd(gen, (offset + n * (width + gap),), getattr(torch, dtype))
    g = whole[offset:].view(n, width + gap)[:, :width]
    ids = _ids(gen, n, rows, kind)
    out = torch.full((rows, width), float("nan"), device="cuda")
    M.mlip_embed_grad(g, ids, rows, out=out)
    assert torch.equal(out.double(), _want(g, ids, rows))


# one row a step (33 columns and more), several; one block, a few, all of them; remainders of the steps of 8 or 16 rows and of the blocks' shares
FEW = [(n, rows, width) for width in (3, 17, 33, 64) for rows in (1, 8, 70) for n in (1, 15, 16, 17, 255, 257, 4095, 16129, 100_003)] + \
      [(300_007, 8, 100), (70_001, 20, 257), (400_009, 3, 2), (1_000_188, 8, 64), (1_000_188, 89, 2)]


@pytest.mark.parametrize("kind", ["even", "hot"])
@pytest.mark.parametrize("n,rows,width", FEW)
def test_few_rows(n, rows, width, kind):
    _check(n, rows, width, "float32", kind)
    _check(n, rows, width, "bfloat16", kind, offset=1, gap=3)


# more than 100 MB, which are read past the caches where rows begin at whole lines: one tile of columns, several of whole lines, several that share lines
@pytest.mark.parametrize("kind", ["even", "hot"])
@pytest.mark.parametrize("n,rows,width,dtype", [(400_003, 8, 64, "float32"), (800_017, 3, 64, "bfloat16"), (280_009, 30, 96, "float32"), (200_003, 60, 128, "float32"),
                                                (70_001, 8, 768, "bfloat16"), (1_600_007, 8, 32, "float16"), (3_300_001, 200, 8, "float32"), (400_003, 8, 65, "float32")])
def test_few_rows_larger_than_the_caches(n, rows, width, dtype, kind):
    _check(n, rows, width, dtype, kind)


@pytest.mark.parametrize("kind", ["even", "hot"])
@pytest.mark.parametrize("n,rows,width", [(1, 300, 5), (2047, 300, 64), (2049, 300, 33), (20_011, 5000, 3), (100_003, 300, 64), (100_003, 9000, 257), (300_007, 14161, 33),
                                          (524_289, 1000, 1), (40_009, 40_000, 130)])
def test_many_rows(n, rows, width, kind):
    _check(n, rows, width, "float32", kind)
    _check(n, rows, width, "bfloat16", kind, offset=1, gap=3)


@pytest.mark.parametrize("kind", ["even", "hot"])
@pytest.mark.parametrize("n,rows,width,dtype", [(400_003, 300, 64, "float32"), (800_017, 3000, 64, "bfloat16"), (110_003, 9000, 256, "float32"), (60_007, 50_021, 1024, "bfloat16"),
                                                (6_400_009, 1000, 8, "bfloat16")])
def test_many_rows_larger_than_the_caches(n, rows, width, dtype, kind):
    _check(n, rows, width, dtype, kind)


@pytest.mark.parametrize("out", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("width", [1, 4, 5, 9, 13, 33, 64, 77, 258])
def test_added_to_old_content(width, dtype, out):
    """Widths whose lots of columns overlap: a column that two lots have is added to once.  Old content and sums are multiples of 1/2 below 2^14."""
    import torch
    import paper_2506_02023_amd as M
    for n, rows in ((300, 6), (2500, 6), (300, 400), (2500, 400), (9001, 700)):
        for kind in ("even", "hot"):
            gen = torch.Generator(device="cuda").manual_seed(n + rows + width)
            g, ids = _odd(gen, (n, width), getattr(torch, dtype)), _ids(gen, n, rows, kind)
            whole = torch.full((rows, width + 4), 9.0, dtype=getattr(torch, out), device="cuda")
            part = whole[:, 1:width + 1]
            part.copy_(torch.randint(-50, 50, (rows, width), generator=gen, device="cuda"))
            want = _want(g, ids, rows, part, 0.5)
            assert float(want.abs().max()) < 2 ** 14
            assert M.mlip_embed_grad(g, ids, rows, 0.5, out=part, accumulate=True) is part
            assert torch.equal(part, want.to(part.dtype)), (n, rows, kind)
            assert (whole[:, 0] == 9).all() and (whole[:, width + 1:] == 9).all()


@pytest.mark.parametrize("n,rows,width", [(3001, 6, 2), (3001, 6, 40), (3001, 700, 2)])
def test_columns_far_apart(n, rows, width):
    """Columns so far apart that a lane's offsets pass 32 bits: (columns, places) transposed, with 2^30 / width places and more"""
    import torch
    import paper_2506_02023_amd as M
    gen = torch.Generator(device="cuda").manual_seed(n + width)
    apart = (1 << 30) // width + 7
    g = torch.zeros((width, apart), dtype=torch.bfloat16, device="cuda")[:, 5:n + 5].t()
    g.copy_(_odd(gen, (n, width), torch.float32))
    assert g.stride() == (1, apart)
    ids = _ids(gen, n, rows, "hot")
    out = M.mlip_embed_grad(g, ids, rows, out=torch.empty((rows, width), device="cuda"))
    assert torch.equal(out.double(), _want(g, ids, rows))
    table = g[:rows]
    out = M.mlip_embed(table, ids, out=torch.empty((n, width), device="cuda"))
    there = (ids >= 0) & (ids < rows)
    assert torch.equal(out[there], table.float()[ids[there].long()]) and (out[ids < 0] == 0).all() and out[ids >= rows].isnan().all()


@pytest.mark.parametrize("width", [33, 64, 90])
@pytest.mark.parametrize("dtype,out", [("float32", "bfloat16"), ("bfloat16", "float32"), ("float16", "float32"), ("float32", "float16")])
def test_large_lookups_into_another_type(width, dtype, out):
    """Results beyond 100 MB of another type than the table's: the fp32 product, rounded to the type, bit for bit, at places that are whole lots and that are not"""
    import torch
    import paper_2506_02023_amd as M
    dt, dt_out = getattr(torch, dtype), getattr(torch, out)
    n = 104_000_000 // (width * dt_out.itemsize)
    gen = torch.Generator(device="cuda").manual_seed(width)
    table = torch.randn((300, width), generator=gen, device="cuda").to(dt)
    species = torch.randint(-3, 300, (n,), generator=gen, device="cuda", dtype=torch.int32)
    want = torch.cat([(table.float() * 1.5).to(dt_out), torch.zeros((1, width), dtype=dt_out, device="cuda")])[torch.where(species < 0, 300, species).long()]
    for offset, gap in ((0, 0), (1, 0), (0, 6), (5, 7)):
        whole = torch.full((offset + n * (width + gap),), 7.0, dtype=dt_out, device="cuda")
        got = whole[offset:].view(n, width + gap)[:, :width]
        M.mlip_embed(table, species, 1.5, out=got)
        assert torch.equal(got, want)
        assert (whole[:offset] == 7).all() and (whole[offset:].view(n, width + gap)[:, width:] == 7).all()
