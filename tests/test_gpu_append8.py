"""Writing into a paged cache of 8 bits, against the same in plain torch: without a rotation bit by bit."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_cache8 as P
from tests.test_gpu_paged import ints
from tests.test_gpu_rotation import close, frequencies

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1234)


class Cache8:
    """Sequences (new rows, keys with them) and a pool of pages that hold what older rows left, or anything."""

    def __init__(self, seqs, Hkv, D, dtype, page=16, hidden=(), pad=0, seed=0, heads_first=False, spread=0.5):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.seqs, self.page, self.dtype, self.D, self.Hkv = seqs, page, dtype, D, Hkv
        T = sum(a for a, _ in seqs) + pad
        kv = rnd(T, 2 * Hkv, D) * torch.exp(spread * rnd(T, 2 * Hkv, 1))
        kv = kv.to(dtype)
        self.k, self.v = kv[:, :Hkv], kv[:, Hkv:]
        need = [-(-n // page) for _, n in seqs]
        self.n_pages = sum(need) + 4
        self.table_host = np.full((len(seqs), max(max(need), 1)), self.n_pages + 3, dtype=np.int32)
        order = iter(np.random.default_rng(seed).permutation(self.n_pages))
        for i, n in enumerate(need):
            self.table_host[i, :n] = [next(order) for _ in range(n)]
        for (i, c), number in dict(hidden).items():
            self.table_host[i, c] = number
        self.table = ints(self.table_host)
        self.codes, self.scales = [], []
        for _ in range(2):
            codes, scales = P.quantised(rnd(self.n_pages, page, Hkv, D) * torch.exp(rnd(self.n_pages, page, Hkv, 1)))
            if heads_first:
                codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
                scales = scales.transpose(0, 1).contiguous().transpose(0, 1)
            self.codes.append(codes)
            self.scales.append(scales)
        self.cu, self.lens = ints(np.cumsum([0] + [a for a, _ in seqs])), ints([n for _, n in seqs])

    def params(self):
        return B.make_kv_append8_params(self.k, self.v, *self.codes, *self.scales, self.cu, self.lens, self.table)

    def plain(self, k=None):
        """What the cache should hold afterwards."""
        codes, scales = [x.clone() for x in self.codes], [x.clone() for x in self.scales]
        for c, s, x in zip(codes, scales, (self.k if k is None else k, self.v)):
            P.append(c, s, x.double(), self.seqs, self.table_host, self.n_pages)
        return codes, scales

    def check(self, want, what):
        torch.cuda.synchronize()
        for name, c, s, wc, ws in zip("kv", self.codes, self.scales, *want):
            assert bool(torch.equal(s, ws)), (what, name, (s != ws).nonzero()[:4].tolist())
            assert P.same_numbers(c, wc), (what, name, (c != wc).nonzero()[:4].tolist())


SEQS = [
    [(1, 1)],
    [(1, 5000)],
    [(16, 16)],
    [(17, 17), (15, 31), (1, 32), (2, 32), (5, 19), (33, 1000)],
    [(40, 50), (1, 16), (1, 17), (3, 9), (5, 2), (0, 30), (0, 0), (1, 0)],
    [(300, 777)],
    [(1, n) for n in range(1, 70)],
]


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (FP32, 128), (FP32, 64)])
@pytest.mark.parametrize("s", range(len(SEQS)))
def test_against_plain_torch(dtype, D, s):
    for n, (page, Hkv) in enumerate([(16, 2), (64, 1), (256, 3)]):
        c = Cache8(SEQS[s], Hkv, D, dtype, page, pad=n, seed=s + n, heads_first=n == 1)
        want = c.plain()
        B.cf_kv_append8(c.params())
        c.check(want, (SEQS[s][:3], page))


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_pages_that_are_none(dtype, D):
    hidden = {(0, 2): -1, (1, 0): 10**9, (2, 0): -2**31, (2, 1): 2**31 - 1}
    c = Cache8([(40, 70), (3, 9), (30, 40), (20, 25)], 2, D, dtype, 16, hidden, pad=2, seed=1)
    want = c.plain()
    B.cf_kv_append8(c.params())
    c.check(want, "hidden")


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_token_by_token(dtype):
    """A block that fills up while its rows grow: its scale grows with them and the older rows are rounded again; shrinking rows leave it."""
    c = Cache8([(1, 1), (1, 1)], 2, 64, dtype, 32, seed=2)
    grown = 0
    for n in range(1, 33):
        size = torch.tensor([1.37 ** n, 1.6 ** -n], device=DEV)[:, None, None]
        fresh = (torch.randn(2, 4, 64, device=DEV) * size).to(dtype)
        c.k.copy_(fresh[:, :2]), c.v.copy_(fresh[:, 2:])
        c.seqs, c.lens = [(1, n), (1, n)], ints([n, n])
        before = [x.clone() for x in c.scales]
        want = c.plain()
        B.cf_kv_append8(c.params())
        c.check(want, n)
        grown += sum(int((a != b).sum()) for a, b in zip(before, c.scales))
    assert grown > 30


def test_values_of_any_size():
    """Zeros, the smallest and the largest numbers, the ends of powers of two, infinities and NaN; a block of zeros that gets others."""
    c = Cache8([(16, 16), (16, 32), (3, 5), (1, 17)], 1, 64, FP32, 16, seed=3)
    T = 36
    x = torch.randn(T, 1, 64, device=DEV)
    x[0:16] = 0
    x[1, 0, 3] = -0.0
    x[16:32] *= 1e-38
    x[16, 0, :4] = torch.tensor([1e-45, 2.0 ** -126, 2.0 ** -120, 0.0], device=DEV)
    x[32:35] *= 1e38
    x[32, 0, :3] = torch.tensor([float("inf"), float("nan"), -float("inf")], device=DEV)
    c.k.copy_(x)
    c.v.copy_(torch.where(torch.arange(64, device=DEV) % 2 == 0, 448.0, 449.0 - 1e-3) * 2.0 ** torch.arange(-18, 18, device=DEV)[:, None, None])
    want = c.plain()
    B.cf_kv_append8(c.params())
    c.check(want, "sizes")
    c2 = Cache8([(15, 15)], 1, 64, FP32, 16, seed=4)
    c2.k.zero_()
    for fresh, n in ((None, 15), (1e-3, 16)):
        if fresh is not None:
            c2.k, c2.v = torch.full((1, 1, 64), fresh, device=DEV), c2.v[:1].contiguous().view(1, 1, 64)
            c2.seqs, c2.lens, c2.cu = [(1, 16)], ints([16]), ints([0, 1])
        want = c2.plain()
        B.cf_kv_append8(c2.params())
        c2.check(want, n)


@pytest.mark.parametrize("content", [float("nan"), float("inf"), -3.0, 0.0, 3e38])
def test_whatever_stood_in_a_scale(content):
    """A block of new rows alone does not look at what its scale was."""
    c = Cache8([(16, 32), (5, 5)], 2, 64, BF16, 16, seed=5)
    want = c.plain()
    for i, p in ((0, 1), (1, 0)):
        for s in c.scales:
            s[int(c.table_host[i, p])] = content
    B.cf_kv_append8(c.params())
    c.check(want, content)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [(BF16, 128, 128), (BF16, 64, 32), (FP32, 128, 80), (FP32, 64, 64)])
def test_with_rotation(dtype, D, rot, interleaved):
    """Keys are rotated in 32 bits and rounded once: half a step of their numbers (2^-4, or 2^-10 of their scale) off the rotated ones in 64."""
    seqs = [(40, 50), (1, 16), (1, 17), (3, 9), (5, 2), (0, 30), (1, 5000), (200, 70000)]
    f = frequencies(rot)
    c = Cache8(seqs, 2, D, dtype, 64, pad=2, seed=6)
    T, pos = 251, torch.cat([torch.arange(n - a, n, device=DEV) for a, n in seqs]).clamp(min=0)
    exactly, tol = P.turn_tolerance(c.k[:T], pos, f, interleaved, False, FP32)
    (codes, v_codes), (scales, v_scales) = c.plain(torch.cat([exactly, exactly[:2]]))
    q = torch.randn(T + 2, 5, D, device=DEV).to(dtype)
    q_out = torch.full_like(q, 7.0)
    B.cf_kv_append8(c.params(), B.make_append_rotation(B.make_rotation(f, interleaved), q, q_out))
    torch.cuda.synchronize()
    want, q_tol = P.turn_tolerance(q[:T], pos, f, interleaved, False, dtype)
    close(q_out[:T], want, q_tol, "queries")
    assert bool((q_out[T:] == 7.0).all())
    assert P.same_numbers(c.codes[1], v_codes) and bool(torch.equal(c.scales[1], v_scales)) and bool(torch.equal(c.scales[0], scales))
    got, held = P.dequantised(c.codes[0], c.scales[0]), P.dequantised(codes, scales)
    new = torch.zeros(c.n_pages, 64, dtype=torch.bool, device=DEV)
    row = 0
    for i, (a, n) in enumerate(seqs):
        for r in range(a):
            j = n - a + r
            if j < 0:
                continue
            at = int(c.table_host[i, j // 64])
            new[at, j % 64] = True
            x = exactly[row + r]
            p = scales[at, :, j % 64 // 16].double()[:, None]
            close(got[at, j % 64], x, torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * p) * (1 + 2.0 ** -20) + 1.07 * tol[row + r], (i, r))
        row += a
    assert bool(torch.equal(got[~new], held[~new]))


def test_many_sequences_and_streams():
    rng = np.random.default_rng(7)
    new = [1, 0, 0, 40] + [1] * 4000 + [0] * 1000 + [3]
    c = Cache8([(a, a + int(b)) for a, b in zip(new, rng.integers(0, 30, len(new)))], 1, 64, BF16, 16, seed=7)
    want = c.plain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.cf_kv_append8(c.params())
    torch.cuda.current_stream().wait_stream(side)
    c.check(want, "many")


def test_a_graph():
    c = Cache8([(1, 20), (2, 500)], 2, 128, BF16, 16, seed=8)
    p = c.params()
    B.cf_kv_append8(p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cf_kv_append8(p)
    for step in range(4):
        c.seqs = [(1, 20 + step), (2, 480 + 3 * step)]
        c.lens.copy_(ints([n for _, n in c.seqs]))
        c.k.copy_(torch.randn(c.k.shape, device=DEV) * 2.0 ** step), c.v.copy_(torch.randn(c.k.shape, device=DEV))
        torch.cuda.synchronize()
        want = c.plain()
        graph.replay()
        c.check(want, step)


def test_pages_beyond_32_bits():
    page, Hkv, D = 256, 8, 128
    n = (5 << 30) // (page * Hkv * D)
    codes = [torch.zeros(n, page, Hkv, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.ones(n, Hkv, page // 16, device=DEV) for _ in range(2)]
    k, v = (torch.randn(20, Hkv, D, device=DEV).to(BF16) for _ in range(2))
    table = ints([[n - 1, n - 2]])
    B.cf_kv_append8(B.make_kv_append8_params(k, v, *codes, *scales, ints([0, 20]), ints([260]), table))
    torch.cuda.synchronize()
    for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
        small_c, small_s = torch.zeros(2, page, Hkv, D, dtype=torch.uint8, device=DEV), torch.ones(2, Hkv, page // 16, device=DEV)
        P.append(small_c, small_s, x.double(), [(20, 260)], np.array([[0, 1]]), 2)
        assert bool(torch.equal(c[n - 1], small_c[0])) and bool(torch.equal(c[n - 2], small_c[1])) and not bool(c[:n - 2].any())
        assert bool(torch.equal(s[n - 2:], small_s.flip(0)))


@pytest.mark.parametrize("D,dtype", [(64, FP32), (128, BF16)])
def test_a_block_keeps_any_larger_scale_and_no_smaller_one(D, dtype):
    """Scales that no append writes: above those that finite elements need the block keeps them, below the least it is rounded to that."""
    for e in (127, 126, 125, 121, 120, -111, -112, -126, -127):
        c = Cache8([(1, 5), (3, 20), (2, 2)], 2, D, dtype, seed=e + 200)
        big = e > 0
        c.k *= 2.0 ** 118 if big else 2.0 ** -116
        c.v *= 2.0 ** 115 if big else 2.0 ** -104
        for s in c.scales:
            s.fill_(0.0 if e == -127 else 2.0 ** e)
        want = [x.clone() for x in c.codes], [s.fill_(2.0 ** e) if e > -127 else s.double().fill_(2.0 ** -127) for s in (x.clone() for x in c.scales)]
        for codes, scales, x in zip(*want, (c.k, c.v)):
            P.append(codes, scales, x.double(), c.seqs, c.table_host, c.n_pages)
        B.cf_kv_append8(c.params())
        torch.cuda.synchronize()
        for got, scales, w, ws in zip(c.codes, c.scales, *want):
            assert P.same_numbers(got, w), e
            kept = ws.double() == 2.0 ** e                   # (what is as it was may be 0 still)
            assert bool(torch.equal(scales[~kept].double(), ws[~kept].double())) and bool((scales[kept] == (0.0 if e == -127 else 2.0 ** e)).all()), e


@pytest.mark.parametrize("D,dtype,interleaved", [(128, BF16, False), (64, BF16, True), (128, FP32, True), (64, FP32, False)])
def test_a_large_call_does_what_its_sequences_calls_do(D, dtype, interleaved):
    """Queries, keys and values of several thousand rows, whose launch is laid out otherwise, against a call for each sequence, bit by bit."""
    seqs = [(1500, 1600), (3, 40), (1, 900), (2600, 2600), (0, 5), (17, 17)]
    T, Hq, pad = sum(a for a, _ in seqs), 14, 3
    one, two = (Cache8(seqs, 2, D, dtype, 64, seed=9, pad=pad) for _ in range(2))
    q = torch.randn(T + pad, Hq, D, device=DEV).to(dtype)
    rotation = B.make_rotation(frequencies(D), interleaved)
    outs = [torch.full_like(q, 7.0) for _ in range(2)]
    B.cf_kv_append8(one.params(), B.make_append_rotation(rotation, q, outs[0]))
    row = 0
    for i, (a, n) in enumerate(seqs):
        if a:
            rows = slice(row, row + a)
            B.cf_kv_append8(B.make_kv_append8_params(two.k[rows], two.v[rows], *two.codes, *two.scales, ints([0, a]), ints([n]), two.table[i:i + 1]),
                            B.make_append_rotation(rotation, q[rows], outs[1][rows]))
        row += a
    torch.cuda.synchronize()
    assert bool(torch.equal(outs[0], outs[1])) and bool((outs[0][T:] == 7.0).all())
    for x, y in zip(one.codes + one.scales, two.codes + two.scales):
        assert bool(torch.equal(x, y))
