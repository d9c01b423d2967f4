"""Windowed and paged calls at shapes where another path begins: thousands of sequences, wide groups of heads, pages that sequences share, the
largest pages, more fp32 workgroups than compute units."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_window as W
from tests.test_gpu_paged import Batch, ints
from tests.test_gpu_window import HUGE, Chunk

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 3), (FP32, 2)])
def test_thousands_of_sequences(dtype, new):
    """Sequences are found 64 bounds at a time: 4200 of them, runs of empty ones, some without a key."""
    rng = np.random.default_rng(4)
    seqs = [(int(rng.integers(0, new + 1)) if i % 700 < 500 else 0, int(rng.integers(0, 40))) for i in range(4200)]
    b = Batch(seqs, 2, 1, 64, dtype, 16, pad=5, seed=13)
    b.check(b.run(), new)


@pytest.mark.parametrize("dtype,D,flags", [(BF16, 128, 0), (BF16, 64, 0), (FP32, 128, 0), (BF16, 128, B.CF_FLAG_SCALAR_KERNELS)])
def test_wide_groups_and_shared_pages(dtype, D, flags):
    """A group's rows are more than a tile of few rows holds; two sequences begin with the same pages."""
    for Hq, Hkv in ((40, 1), (64, 1), (130, 2)):
        b = Batch([(1, 700), (1, 300), (2, 40), (9, 320)], Hq, Hkv, D, dtype, 32, window=250, sinks=20, seed=14)
        for i, columns in ((1, 8), (3, 5)):
            b.table_host[i, :columns] = b.table_host[0, :columns]
            for mine, first in zip(b.keys[i], b.keys[0]):
                mine[:32 * columns] = first[:32 * columns]
        b.table = ints(b.table_host)
        b.check(b.run(flags), (Hq, Hkv))


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (FP32, 64)])
def test_the_largest_pages(dtype, D):
    b = Batch([(1, 70000), (3, 10), (40, 65536)], 2, 1, D, dtype, 65536, seed=15)
    b.check(b.run(), "largest pages")


@pytest.mark.parametrize("D", [64, 128])
def test_fp32_chunks_of_many_workgroups(D):
    segs = [(300, 40), (1, 0), (17, 100), (700, 0)]
    c = Chunk(segs, 8, 2, D, FP32, seed=16)
    for window, sinks in ((1, 0), (60, 3), (333, 20), (HUGE, 0)):
        c.check(c.run(window, sinks), c.reference(window, sinks), (window, sinks))
    # One value of the first segment's key 70 (position 70, rows 30 .. 79 see it).  Other rows of its block are done again pair by pair: they hold
    # the definition's values, not the same bits.
    ref = c.reference(50, 0)
    tol = W.tolerances(ref, FP32, D, False)
    c.v[70, 1, 3] = float("nan")
    got = c.run(50, 0, backward=False)
    seen = torch.zeros(c.o.shape, dtype=torch.bool, device=c.o.device)
    seen[30:80, 4:] = True
    W.check(dict(o=got["o"][~seen], lse=got["lse"]), dict(o=ref["o"][~seen], lse=ref["lse"]), dict(o=tol["o"][~seen], lse=tol["lse"]), "rows that do not see it")
    rows = got["o"][30:80, 4:]
    assert bool(rows[..., 3].isnan().all()) and bool(torch.cat([rows[..., :3], rows[..., 4:]], -1).isfinite().all())


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128)])
def test_short_slices_behind_long_windows(dtype, D):
    """dQ from parts of the keys: parts that end inside the sinks' and the window's tiles, rows near the beginning, a segment of one row, results
    that repeat bit for bit and a value that is not finite in one row's dO."""
    segs = [(27, 4000), (1, 2500), (40, 10), (65, 700)]
    for Hq, Hkv in ((7, 1), (4, 4)):
        c = Chunk(segs, Hq, Hkv, D, dtype, seed=17)
        for window, sinks in ((3000, 100), (129, 0), (HUGE, 0), (1000, 1500)):
            got = c.run(window, sinks)
            c.check(got, c.reference(window, sinks), (Hq, window, sinks))
            assert bool(torch.equal(got["dq"], c.run(window, sinks)["dq"]))
    clean = c.run(3000, 100)
    c.d_o[5, 1, 7] = float("inf")
    got = c.run(3000, 100)
    others = torch.ones(clean["dq"].shape[:2], dtype=torch.bool, device=c.o.device)
    others[5, 1] = False
    assert bool(torch.equal(got["dq"][others], clean["dq"][others])) and not bool(got["dq"][5, 1].isfinite().all())


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("segs", [[(400, 50), (1, 0), (180, 300)], [(900, 50), (1, 0), (300, 700), (129, 0)]])
def test_chunks_of_more_rows(dtype, D, segs):
    """Too many rows for tiles of 16, and for the wavefronts to share keys at all; then one value of the first segment's key 70."""
    c = Chunk(segs, 16, 2, D, dtype, seed=18)
    for window, sinks in ((1, 0), (100, 4), (130, 70), (700, 129), (HUGE, 0)):
        c.check(c.run(window, sinks, tiles=window == 100), c.reference(window, sinks), (window, sinks))
    ref = c.reference(50, 0)
    tol = W.tolerances(ref, dtype, D, True)
    c.v[70, 1, 3] = float("inf")
    got = c.run(50, 0, backward=False)
    seen = torch.zeros(c.o.shape, dtype=torch.bool, device=c.o.device)
    seen[20:70, 8:] = True                           # (position 70, behind 50: rows 20 .. 69 see it)
    W.check(dict(o=got["o"][~seen], lse=got["lse"]), dict(o=ref["o"][~seen], lse=ref["lse"]), dict(o=tol["o"][~seen], lse=tol["lse"]), "rows that do not see it")
    rows = got["o"][20:70, 8:]
    assert bool((rows[..., 3] == float("inf")).all()) and bool(torch.cat([rows[..., :3], rows[..., 4:]], -1).isfinite().all())


@pytest.mark.parametrize("D", [64, 128])
def test_longer_slices_behind_long_windows(D):
    """dQ from parts with the matrix instruction of larger calls; a value that nobody sees changes nothing."""
    c = Chunk([(600, 2500), (300, 20)], 16, 2, D, BF16, seed=19)
    for window, sinks in ((2000, 4), (HUGE, 0), (700, 900)):
        got = c.run(window, sinks)
        c.check(got, c.reference(window, sinks), (window, sinks))
        assert bool(torch.equal(got["dq"], c.run(window, sinks)["dq"]))
    clean = c.run(1500, 0)
    c.k[100, 1, 5] = float("inf")                    # (position 100: no row of the first segment sees it, whose rows begin at 2500)
    got = c.run(1500, 0)
    assert bool(torch.equal(got["o"], clean["o"])) and bool(torch.equal(got["dq"], clean["dq"]))
