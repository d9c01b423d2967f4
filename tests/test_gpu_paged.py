"""Attention over a paged cache and writing into it, on the GPU, against the definition in 64 bits (tests/plain_window.py)."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_window as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32
SCALAR = B.CF_FLAG_SCALAR_KERNELS
KINDS = [(FP32, 64, 0), (FP32, 128, 0), (BF16, 64, 0), (BF16, 128, 0), (BF16, 128, SCALAR), (FP32, 64, SCALAR)]
NAN = float("nan")


def ints(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


class Batch:
    """Sequences (new rows, keys with them), their pages in any order among unused ones; what nobody has written is NaN.  hidden: {(sequence,
    column): number}; pad: rows behind the last sequence; heads_first: pages of [heads][tokens]."""

    def __init__(self, seqs, Hq, Hkv, D, dtype, page=16, window=0, sinks=0, hidden=(), pad=0, columns=0, seed=0, heads_first=False, scale=None,
                 far=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=FP32).to(dtype)
        self.seqs, self.D, self.dtype, self.page, self.window, self.sinks = seqs, D, dtype, page, window, sinks
        self.scale, self.pad = 1 / np.sqrt(D) if scale is None else scale, pad
        T = sum(a for a, _ in seqs)
        qkv = rnd(T + pad, Hq + 2 * Hkv, D)
        self.q, self.k, self.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        need = [-(-n // page) for _, n in seqs]
        n_pages = sum(need) + 5 + far
        table = np.full((len(seqs), max(max(need), 1) + columns), n_pages + 7, dtype=np.int32)
        order = iter(far + np.random.default_rng(seed).permutation(n_pages - far))
        for i, n in enumerate(need):
            table[i, :n] = [next(order) for _ in range(n)]
        for (i, c), number in dict(hidden).items():
            table[i, c] = number
        self.table_host = table
        self.table = ints(np.pad(table, ((0, 0), (0, 3))))[:, :table.shape[1]]
        shape = (n_pages, Hkv, page, D) if heads_first else (n_pages, page, Hkv, D)
        make = lambda: torch.empty(shape, device=DEV, dtype=dtype) if far else torch.full(shape, NAN, device=DEV, dtype=dtype)
        self.kp, self.vp = (x.transpose(1, 2) if heads_first else x for x in (make(), make()))
        self.n_pages = n_pages
        self.keys = [(rnd(n, Hkv, D), rnd(n, Hkv, D)) for _, n in seqs]
        row = 0
        for i, (a, n) in enumerate(seqs):            # older keys; the new rows' own come from k, v
            b = min(a, n)
            self.keys[i][0][n - b:], self.keys[i][1][n - b:] = self.k[row + a - b:row + a], self.v[row + a - b:row + a]
            for j0 in range(0, n - b, page):
                at, m = int(table[i, j0 // page]), min(page, n - b - j0)
                if 0 <= at < n_pages:
                    self.kp[at, :m], self.vp[at, :m] = self.keys[i][0][j0:j0 + m], self.keys[i][1][j0:j0 + m]
            row += a
        self.cu, self.lens = ints(np.cumsum([0] + [a for a, _ in seqs])), ints([n for _, n in seqs])
        self.o = torch.full((T + pad, Hq, D), 7.0, device=DEV, dtype=dtype)
        self.lse = torch.full((Hq, T + pad), 7.0, device=DEV)

    def params(self, flags=0, max_kv_len=0, workspace=None):
        return B.make_paged_params(self.q, self.kp, self.vp, self.o, self.lse, self.cu, self.lens, self.table, self.scale, max_kv_len, self.window,
                                   self.sinks, flags, workspace)

    def append(self):
        B.cf_kv_append(B.make_kv_append_params(self.k, self.v, self.kp, self.vp, self.cu, self.lens, self.table))

    def run(self, flags=0, max_kv_len=0):
        self.append()
        B.cf_attn_paged_fwd(self.params(flags, max_kv_len))
        torch.cuda.synchronize()
        return dict(o=self.o.clone(), lse=self.lse.clone())

    def reference(self):
        Hq, Hkv = self.q.shape[1], self.k.shape[1]
        ref = dict(o=torch.full(self.o.shape, 7.0, dtype=torch.float64, device=DEV), lse=torch.full(self.lse.shape, 7.0, dtype=torch.float64, device=DEV),
                   o_abs=torch.zeros(self.o.shape, dtype=torch.float64, device=DEV))
        row, worst = 0, 0.0
        for i, (a, n) in enumerate(self.seqs):
            held = torch.tensor([0 <= self.table_host[i, j // self.page] < self.n_pages for j in range(n)], dtype=torch.bool, device=DEV)
            p, j = torch.arange(n - a, n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
            seen = (j <= p) & held[None]
            if self.window:
                seen &= (j > p - self.window) | (j < self.sinks)
            for h in range(Hq):
                if n == 0:
                    r = dict(o=0.0, o_abs=0.0, lse=-float("inf"), score_abs=0.0)
                else:
                    k, v = (x[:, h // (Hq // Hkv)].double() for x in self.keys[i])
                    r = W.attention(self.q[row:row + a, h].double(), k, v, self.scale, seen) if a else dict(score_abs=0.0)
                worst = max(worst, r["score_abs"])
                if a:
                    ref["o"][row:row + a, h], ref["o_abs"][row:row + a, h], ref["lse"][h, row:row + a] = r["o"], r["o_abs"], r["lse"]
            row += a
        ref.update(keys=max(max(n for _, n in self.seqs), 1), rows=1, score_abs=worst)
        return ref

    def check(self, got, what):
        ref = self.reference()
        W.check(got, ref, W.tolerances(ref, self.dtype, self.D, self.dtype == BF16), what)


SEQS = [
    [(1, 1)],
    [(1, 5000)],
    [(1, 17), (0, 40), (3, 3), (5, 2), (130, 700), (1, 0), (0, 0), (2, 64)],
    [(1, n) for n in (1, 15, 16, 17, 63, 64, 65, 300, 1000, 2049)],
    [(300, 300)],
    [(7, 3000), (9, 40)],
]


@pytest.mark.parametrize("dtype,D,flags", KINDS)
@pytest.mark.parametrize("s", range(len(SEQS)))
def test_against_the_definition(dtype, D, flags, s):
    for n, (page, Hq, Hkv) in enumerate([(16, 4, 2), (64, 7, 1), (256, 3, 3), (32, 16, 1)]):
        b = Batch(SEQS[s], Hq, Hkv, D, dtype, page, pad=n, columns=n, seed=s + n, heads_first=n == 1)
        b.check(b.run(flags, max_kv_len=[0, 5000, 1, 100][n]), (SEQS[s], page, Hq, Hkv))


@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_windows_and_pages_that_were_given_back(dtype, D, flags):
    """Pages behind the windows of all rows are marked, and their content is gone."""
    for n, (window, sinks, page) in enumerate([(1, 0, 16), (64, 4, 16), (65, 64, 32), (500, 1, 128), (2000, 0, 16), (40, 200, 64), (2**31 - 1, 1000, 16)]):
        seqs = [(1, 1500), (33, 900), (1, 30), (200, 200), (2, 130)]
        hidden = {(i, c): -1 for i, (a, m) in enumerate(seqs) for c in range(-(-m // page)) if (c + 1) * page <= m - a - window + 1 and c * page >= sinks}
        assert n not in (1, 3) or len(hidden) > 5
        b = Batch(seqs, 4, 2, D, dtype, page, window, sinks, hidden, seed=n)
        b.check(b.run(flags), (window, sinks, page))


@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_pages_that_are_none(dtype, D, flags):
    """Any number outside the pages hides its keys: in the middle, at the end (the new rows' own: they are not written), all of them."""
    hidden = {(0, 1): -1, (0, 5): 10**6, (1, 0): 2**31 - 1, (2, 3): -2**31, (2, 4): -5, (3, 0): -1, (3, 1): -1}
    seqs = [(40, 130), (3, 10), (20, 80), (2, 32), (1, 200)]
    b = Batch(seqs, 6, 2, D, dtype, 16, hidden=hidden, seed=3)
    got = b.run(flags)
    b.check(got, "hidden pages")
    assert (got["o"][43 + 20:43 + 22] == 0).all() and torch.isinf(got["lse"][:, 63:65]).all() and (got["o"][40:43] == 0).all()


@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 20), (60, 3)])
@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_lengths_beyond_the_table(dtype, D, flags, window, sinks):
    """kv_lens may promise more keys than the table has columns for; those are hidden."""
    b = Batch([(4, 100), (1, 64), (40, 300)], 4, 2, D, dtype, 16, window, sinks, seed=4)
    b.append()
    narrow = b.table[:, :3]                          # 48 keys of each
    p = B.make_paged_params(b.q, b.kp, b.vp, b.o, b.lse, b.cu, b.lens, narrow, b.scale, window=window, n_sinks=sinks, flags=flags)
    B.cf_attn_paged_fwd(p)
    torch.cuda.synchronize()
    b.table_host = b.table_host.copy()
    b.table_host[:, 3:] = -1
    b.check(dict(o=b.o, lse=b.lse), "narrow table")


@pytest.mark.parametrize("value", [NAN, float("inf")])
@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_what_is_not_finite_reaches_the_rows_that_see_it(dtype, D, flags, value):
    b = Batch([(60, 200), (1, 90)], 4, 2, D, dtype, 32, window=50, seed=5)
    good = b.run(flags)
    for which in ("kp", "vp"):
        x = getattr(b, which)
        at = (int(b.table_host[0, 160 // 32]), 160 % 32, 1, 3)       # key 160: rows at positions 160 .. 199, i.e. 20 .. 59
        keep = x[at].clone()
        x[at] = value
        B.cf_attn_paged_fwd(b.params(flags))
        torch.cuda.synchronize()
        for rows in (slice(0, 20), slice(60, 61)):
            assert torch.allclose(b.o[rows].float(), good["o"][rows].float(), atol=2.0 ** -6 if dtype == BF16 else 1e-5, rtol=0)
            assert torch.isfinite(b.lse[:, rows]).all()
        assert torch.isfinite(b.o[:, :2]).all()
        if which == "vp":
            assert not torch.isfinite(b.o[20:60, 2:, 3]).any() and torch.isfinite(b.o[20:60, 2:, 4:]).all()
        x[at] = keep


@pytest.mark.parametrize("dtype,D", [(FP32, 64), (BF16, 64), (BF16, 128)])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.5])
def test_other_scales(dtype, D, scale):
    b = Batch([(1, 400), (50, 90)], 4, 2, D, dtype, 16, seed=6, scale=scale)
    b.check(b.run(), scale)


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_offsets_beyond_32_bits(dtype, D):
    """Pages that lie more than 2^32 bytes from the first."""
    page, Hkv = 256, 8
    far = (5 << 30) // (page * Hkv * D * (2 if dtype == BF16 else 4))
    b = Batch([(1, 3000), (70, 500)], 16, Hkv, D, dtype, page, seed=7, far=far)
    b.check(b.run(), "far pages")


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (FP32, 64)])
def test_runs_repeat_and_do_not_need_lse(dtype, D):
    b = Batch([(1, 4000), (30, 2500), (1, 7)], 8, 2, D, dtype, 64, seed=8)
    one, two = b.run(), b.run()
    assert bool(torch.equal(one["o"], two["o"])) and bool(torch.equal(one["lse"], two["lse"]))
    p = B.make_paged_params(b.q, b.kp, b.vp, b.o, None, b.cu, b.lens, b.table, b.scale)
    b.o.zero_()
    B.cf_attn_paged_fwd(p)
    torch.cuda.synchronize()
    assert bool(torch.equal(b.o, one["o"]))


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_graphs_of_growing_sequences(dtype, D):
    """One token after the other through one captured graph: lengths, rows and tables change in place; two graphs share a workspace, one
    behind the other; eager work on the same buffers in between."""
    b = Batch([(1, 700), (1, 33), (1, 2)], 8, 2, D, dtype, 16, columns=3, seed=9)
    b.table_host[:, -3:] = [[1, 2, 3]] * 3           # (not reached)
    other = Batch([(2, 900)], 8, 2, D, dtype, 16, seed=10)
    other.append()
    need = max(B.cf_attn_paged_workspace_bytes(x.params(max_kv_len=800)) for x in (b, other))
    ws = torch.zeros(max(need, 256), dtype=torch.uint8, device=DEV)
    p, q = (x.params(max_kv_len=800, workspace=ws) for x in (b, other))
    graphs = []
    for call in ((lambda: (b.append(), B.cf_attn_paged_fwd(p))), (lambda: B.cf_attn_paged_fwd(q))):
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for step in range(4):
        b.seqs = [(1, n + step) for n in (700, 33, 2)]
        b.lens.copy_(ints([n for _, n in b.seqs]))
        fresh = torch.randn(b.q.shape[0], b.q.shape[1] + 4, D, device=DEV).to(dtype)
        b.q.copy_(fresh[:, :8]), b.k.copy_(fresh[:, 8:10]), b.v.copy_(fresh[:, 10:])
        if step:
            b.keys = [tuple(torch.cat([x, new[i:i + 1]]) for x, new in zip(b.keys[i], (b.k, b.v))) for i in range(3)]
        else:
            b.keys = [tuple(torch.cat([x[:-1], new[i:i + 1]]) for x, new in zip(b.keys[i], (b.k, b.v))) for i in range(3)]
        b.o.fill_(1), other.o.fill_(1), ws.fill_(255)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        b.check(dict(o=b.o, lse=b.lse), step)
        other.check(dict(o=other.o, lse=other.lse), step)


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (FP32, 128)])
def test_append_writes_the_new_rows_and_nothing_else(dtype, D):
    """Across page ends, into the middle of a page, with positions before the first, pages that are none and padded rows."""
    hidden = {(0, 2): -1, (3, 0): 10**9}
    b = Batch([(40, 50), (1, 16), (1, 17), (3, 9), (5, 2), (0, 30), (0, 0)], 4, 2, D, dtype, 16, hidden=hidden, pad=3, seed=11)
    for x in (b.kp, b.vp):
        x.copy_(torch.randn(x.shape, device=DEV).to(dtype))
    want = [x.clone() for x in (b.kp, b.vp)]
    row = 0
    for i, (a, n) in enumerate(b.seqs):
        for r in range(a):
            j = n - a + r
            at = int(b.table_host[i, j // 16]) if j >= 0 else -1
            if 0 <= at < b.n_pages:
                for w, new in zip(want, (b.k, b.v)):
                    w[at, j % 16] = new[row + r]
        row += a
    b.append()
    torch.cuda.synchronize()
    assert bool(torch.equal(b.kp, want[0])) and bool(torch.equal(b.vp, want[1]))


def test_another_stream():
    b = Batch([(1, 4000), (64, 900)], 8, 2, 128, BF16, 64, seed=12)
    want = b.run()
    side = torch.cuda.Stream()
    b.o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.append()
        p = b.params()
        B.cf_attn_paged_fwd(p)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert bool(torch.equal(b.o, want["o"]))
