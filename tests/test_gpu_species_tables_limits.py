"""Calls whose kernels need 2^32 threads and more, of which one launch runs only what is left over modulo 2^32: they are made of several launches.

The gradients are one row of small whole numbers for all atoms (an expanded tensor), so every sum is a whole number below 2^24, exact in fp32."""
import pytest

pytestmark = pytest.mark.gpu


def _check(n, rows, width, offset, dtype):
    import torch
    import paper_2506_02023_amd as M
    gen = torch.Generator(device="cuda").manual_seed(rows)
    row = torch.randint(1, 4, (offset + width,), generator=gen, device="cuda").to(dtype)[offset:]
    species = torch.randint(0, rows, (n,), generator=gen, device="cuda", dtype=torch.int32)
    counts = torch.bincount(species, minlength=rows)
    assert int(counts.max()) * 3 < 2 ** 24
    out = M.mlip_embed_grad(row.expand(n, width), species, rows, out=torch.full((rows, width), float("nan"), device="cuda"))
    for r in range(rows):
        assert torch.equal(out[r], row.float() * counts[r]), r


def test_join_of_very_wide_tables():
    """80 rows of 2^20 columns in two blocks of rows: 1024 threads of the join to 16 of the 80 * 2^20 elements"""
    import torch
    _check(3025, 80, 2 ** 20, 0, torch.float32)


@pytest.mark.parametrize("offset", [0, 1])
def test_sums_of_very_many_tiles(offset):
    """257 blocks of rows for each of 16,384 tiles of columns, with tiles grouped by the lines they share (offset 1) and not"""
    import torch
    _check(256 * 16128 + 5, 1, 2 ** 20, offset, torch.bfloat16)
