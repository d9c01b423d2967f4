"""Attention over a paged cache of 8 bits where calls are unlike the others: thousands of sequences, wide groups, shared pages, the largest pages, queries that
are not finite, a batch of padding, how a call is cut, tables of other devices."""
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_cache8 as P
from tests import plain_window as W
from tests.test_gpu_paged import ints
from tests.test_gpu_paged8 import Batch8, KINDS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(5)


@pytest.mark.parametrize("dtype,D", [(FP32, 64), (BF16, 64), (BF16, 128)])
def test_thousands_of_sequences(dtype, D):
    seqs = [(1, n % 37 + 1) for n in range(3000)] + [(0, 5)] * 500 + [(1, 100), (3, 70)]
    b = Batch8(seqs, 2, 1, D, dtype, 16, seed=1)
    got = b.run(max_kv_len=100)
    for i in list(range(0, 3000, 97)) + [3500, 3501]:
        row, (a, n) = int(b.cu[i]), seqs[i]
        k, v = (x[:, 0].double() for x in b.keys[i])
        for h in range(2):
            ref = W.attention(b.q[row:row + a, h].double(), k, v, b.scale, W.visible(a, n, 0, 0, DEV))
            ref.update(keys=n, rows=1)
            W.check(dict(o=got["o"][row:row + a, h], lse=got["lse"][h, row:row + a]), ref, W.tolerances(ref, dtype, D, dtype == BF16), i)


@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_wide_groups(dtype, D, flags):
    for Hq, Hkv, seqs in ((40, 1, [(1, 300), (2, 90)]), (48, 3, [(1, 1000), (1, 3), (7, 7)]), (17, 17, [(1, 65), (5, 64)])):
        b = Batch8(seqs, Hq, Hkv, D, dtype, 32, seed=2)
        b.check(b.run(flags), (Hq, Hkv))


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_shared_pages(dtype, D):
    """A prompt's pages in the tables of several sequences, the same page twice in one."""
    b = Batch8([(1, 200), (1, 200), (2, 130)], 8, 2, D, dtype, 16, seed=3)
    b.table_host = b.table_host.copy()
    b.table_host[1, :8] = b.table_host[0, :8]
    b.table_host[2, 3] = b.table_host[2, 2]
    b.table.copy_(ints(b.table_host))
    b.read()
    b.check(b.run(), "shared")


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (FP32, 128)])
@pytest.mark.parametrize("page", [65536, 1024])
def test_the_largest_pages(dtype, D, page):
    b = Batch8([(1, 70000 if page == 65536 else 3000), (40, 100)], 4, 2, D, dtype, page, seed=4)
    b.check(b.run(), page)


@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_queries_that_are_not_finite(dtype, D, flags, value):
    """Their row and head, and no others."""
    b = Batch8([(60, 200), (1, 90), (200, 300)], 4, 2, D, dtype, 32, seed=5)
    good = b.run(flags)
    for row, h in ((7, 1), (60, 3), (150, 0)):
        b.q[row, h, 5] = value
    got = b.run(flags)
    hit = torch.zeros(b.o.shape[:2], dtype=torch.bool, device=DEV)
    for row, h in ((7, 1), (60, 3), (150, 0)):
        hit[row, h] = True
    assert not torch.isfinite(got["o"][hit]).any() and not torch.isfinite(got["lse"].t()[hit]).any()
    assert bool(torch.equal(got["o"][~hit], good["o"][~hit])) and bool(torch.equal(got["lse"].t()[~hit], good["lse"].t()[~hit]))


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_a_batch_of_padding(dtype, D):
    """No sequence has a row: nothing is written."""
    b = Batch8([(0, 20), (0, 0)], 4, 2, D, dtype, 16, pad=5, seed=6)
    got = b.run()
    assert bool((got["o"] == 7.0).all()) and bool((got["lse"] == 7.0).all())


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (FP32, 64)])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_the_ends_of_parts_and_tiles(dtype, D, page):
    """Lengths around multiples of 16, 64 and of a part's keys, one call for all and one for each: the same attention however it is cut."""
    lens = [n + d for n in (16, 64, 256, 512, 1024) for d in (-1, 0, 1)] + [1, 2, 5000]
    b = Batch8([(1, n) for n in lens], 8, 2, D, dtype, page, seed=7)
    for hint in (0, 5000, 64, 100000):
        b.o.fill_(7), b.lse.fill_(7)
        b.check(b.run(max_kv_len=hint), (page, hint))
    for n in (513, 1025, 5000):
        one = Batch8([(1, n)], 8, 2, D, dtype, page, seed=n)
        one.check(one.run(max_kv_len=n), n)


def test_a_workspace_that_is_too_small():
    b = Batch8([(1, 20000)], 8, 2, 128, BF16, 64, seed=8)
    p = b.params(max_kv_len=20000)
    need = B.cf_attn_paged8_workspace_bytes(p)
    assert need > 0 and p.a.workspace_bytes >= need
    p.a.workspace_bytes = need - 1
    with pytest.raises(B.CfError) as e:
        B.cf_attn_paged8_fwd(p)
    assert e.value.code == B.CF_EINVAL
    p.a.workspace_bytes, p.a.workspace = need, p.a.workspace + 8
    with pytest.raises(B.CfError):
        B.cf_attn_paged8_fwd(p)


def test_older_rows_of_a_block_are_as_the_attention_reads_them():
    """Appends that raise a block's scale change what later queries see of its older rows by their rounding, no more.  Half a step of a number is 2^-4 of
    it, or 2^-10 scales where it is subnormal; numbers that stay normal under a larger scale are not rounded again, and the half steps of the scales that
    made it subnormal double from one to the next: both together are at most twice the larger of the two."""
    D, page = 64, 16
    codes = [torch.zeros(2, page, 1, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.ones(2, 1, 1, device=DEV) for _ in range(2)]
    table, rows = ints([[1]]), []
    for n in range(1, 17):
        k, v = (torch.randn(1, 1, D, device=DEV) * 2.0 ** (n // 3) for _ in range(2))
        rows.append((k[0], v[0]))
        B.cf_kv_append8(B.make_kv_append8_params(k, v, *codes, *scales, ints([0, 1]), ints([n]), table))
        torch.cuda.synchronize()
        for i, (c, s) in enumerate(zip(codes, scales)):
            got = P.values(c[1, :n, 0], s[1, 0, 0])
            want = torch.stack([r[i][0] for r in rows]).double()
            assert bool(((got - want).abs() <= 2 * torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * s[1, 0, 0].double())).all()), n


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("seqs,Hq,Hkv,columns", [([(1, 900), (1, 40), (3, 3), (2, 500), (0, 7)], 8, 2, 200000),      # (rows of the table for 3 M keys and more)
                                                 ([(2, 300), (2, 77), (1, 1)], 14, 1, 0), ([(2, 600), (2, 130)], 36, 3, 0)])
def test_tiles_of_32_rows_at_head_dim_64(seqs, Hq, Hkv, columns, page):
    """What the host takes for long calls, and sequences of 17 to 32 rows."""
    b = Batch8(seqs, Hq, Hkv, 64, BF16, page, columns=columns, pad=2, seed=page)
    for hint in (0, max(n for _, n in seqs)):
        b.o.fill_(7), b.lse.fill_(7)
        b.check(b.run(max_kv_len=hint), (page, hint))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 6, 8])
def test_pairs_of_heads(dtype, Hkv):
    """Heads one by one and two by two, any number of workgroups; a call with itself again."""
    for seqs in ([(1, 100)], [(1, 70), (2, 300), (1, 5)], [(1, 40 * n + 1) for n in range(9)], [(40, 90), (1, 1000)]):
        b = Batch8(seqs, 2 * Hkv, Hkv, 64, dtype, 32, seed=Hkv)
        got, again = b.run(), b.run()
        b.check(got, (seqs[:2], Hkv))
        assert bool(torch.equal(got["o"], again["o"])) and bool(torch.equal(got["lse"], again["lse"]))
