"""Windowed attention with sinks on the GPU against its definition in 64 bits (tests/plain_window.py), element by element."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from paper_2503_02356_amd.runner import ChunkAttention
from tests import plain_window as W
from tests import parity as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32
SCALAR, ONE = B.CF_FLAG_SCALAR_KERNELS, B.CF_FLAG_DKV_SINGLE_WRITER
KINDS = [(FP32, 64, 0), (FP32, 128, 0), (BF16, 64, 0), (BF16, 128, 0), (BF16, 128, ONE), (BF16, 64, SCALAR), (FP32, 128, SCALAR)]
HUGE = 2**31 - 1


def ints(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


class Chunk:
    """Inputs of a chunk of segments (lq, prefix); strided: q, k, v are views of one buffer, the results views of wider ones."""

    def __init__(self, segs, Hq, Hkv, D, dtype, seed=0, strided=False, scale=None):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=FP32).to(dtype)
        self.segs, self.D, self.dtype, self.scale = segs, D, dtype, 1 / np.sqrt(D) if scale is None else scale
        T, Tk = sum(a for a, _ in segs), sum(a + b for a, b in segs)
        wide = 8 if strided else 0
        view = lambda n, H: rnd(n, H + (1 if strided else 0), D + wide)[:, :H, :D]
        self.q, self.d_o = view(T, Hq), view(T, Hq)
        kv = rnd(Tk, 2 * Hkv, D + wide)[:, :, :D]
        self.k, self.v = kv[:, :Hkv], kv[:, Hkv:]
        self.o, self.dq = view(T, Hq), view(T, Hq)
        self.lse = torch.full((Hq, T), 3.0, device=DEV)
        self.start = torch.randn(2, Tk, Hkv, D, generator=g, device=DEV)
        self.cu_q, self.cu_k = ints(np.cumsum([0] + [a for a, _ in segs])), ints(np.cumsum([0] + [a + b for a, b in segs]))

    def run(self, window, sinks, flags=0, tiles=False, backward=True):
        table = ints(B.cf_attn_q_tiles(self.cu_q.cpu().numpy(), self.cu_k.cpu().numpy())) if tiles else None
        fp = B.make_fwd_params(self.q, self.k, self.v, self.o, self.lse, self.cu_q, self.cu_k, self.scale, flags, q_tiles=table)
        B.cf_attn_window_fwd(fp, window, sinks)
        got = dict(o=self.o.clone(), lse=self.lse.clone())
        if backward:
            dkv = self.start.clone()
            ws = torch.empty(B.cf_attn_window_bwd_workspace_bytes(fp, window, sinks), dtype=torch.uint8, device=DEV)
            B.cf_attn_window_bwd(B.make_bwd_params(fp, self.d_o, self.dq, dkv[0], dkv[1], ws), window, sinks)
            got.update(dq=self.dq.clone(), dk=dkv[0], dv=dkv[1])
        torch.cuda.synchronize()
        return got

    def reference(self, window, sinks):
        return W.chunk(self.q, self.k, self.v, self.scale, self.segs, window, sinks, self.d_o)

    def check(self, got, ref, what):
        tol = W.tolerances(ref, self.dtype, self.D, self.dtype == BF16)
        ref = dict(ref)
        if "dk" in got:                              # added to what stood there: one more rounding to fp32
            for n, name in enumerate(("dk", "dv")):
                ref[name] = ref[name] + self.start[n].double()
                tol[name] = tol[name] + 2.0 ** -23 * ref[name].abs() + 2.0 ** -24 * self.start[n].double().abs()
        W.check(got, ref, tol, what)


GEOMETRIES = [
    # segments (queries, prefix), windows and sinks
    ([(1, 0)], [(1, 0), (5, 3)]),
    ([(1, 513)], [(1, 0), (64, 4), (300, 70), (514, 0)]),
    ([(300, 0), (1, 0), (63, 0), (129, 0), (64, 5)], [(1, 0), (1, 1), (7, 3), (64, 64), (65, 0), (HUGE, 0), (100, HUGE)]),
    ([(200, 700)], [(100, 4), (333, 130), (64, 700), (899, 1), (31, 0)]),
    ([(5, 1000), (130, 0), (2, 2), (257, 129)], [(32, 1), (128, 16), (200, 200)]),
    # rows far behind the sinks: several pieces, near rows that end inside one, no near rows, sinks that fill more than a piece's keys
    ([(900, 50), (400, 0), (513, 1000), (1, 0)], [(30, 20), (100, 2), (5, 300), (190, 1)]),
    ([(1024, 0)], [(100, 4), (257, 33), (16, 16)]),
]


@pytest.mark.parametrize("dtype,D,flags", KINDS)
@pytest.mark.parametrize("g", range(len(GEOMETRIES)))
def test_against_the_definition(dtype, D, flags, g):
    segs, masks = GEOMETRIES[g]
    for n, (window, sinks) in enumerate(masks):
        Hq, Hkv = [(4, 2), (7, 1), (3, 3)][(n + g) % 3]
        c = Chunk(segs, Hq, Hkv, D, dtype, seed=10 * g + n, strided=n % 2 == 1)
        ref = c.reference(min(window, 10**6), min(sinks, 10**6))
        c.check(c.run(window, sinks, flags, tiles=n % 3 == 2), ref, (segs, window, sinks, Hq, Hkv))


@pytest.mark.parametrize("dtype,D,limit", [(FP32, 64, 2e-6), (FP32, 128, 2e-6), (BF16, 64, 3e-3), (BF16, 128, 3e-3)])
def test_relative_errors(dtype, D, limit):
    """2-norms.  bf16: a result and a product rounded to half a step at most, 2^-8 of the value, 0.42 of that in the mean of squares
    (mantissas spread over a binade): 1.65e-3 each, 2.4e-3 both.  fp32: some 20 roundings of 2^-24 in a row."""
    c = Chunk([(700, 900), (90, 0)], 8, 2, D, dtype, seed=4)
    ref, got = c.reference(300, 4), c.run(300, 4)
    for n, name in enumerate(("o", "lse", "dq", "dk", "dv")):
        g = got[name].double() - (c.start[n - 3].double() if n > 2 else 0)
        rel = float((g - ref[name]).norm() / ref[name].norm())
        print(dtype, D, name, rel)
        assert rel < (2e-6 if name == "lse" else limit), (name, rel)


@pytest.mark.parametrize("dtype,D", [(FP32, 64), (BF16, 64), (BF16, 128)])
def test_a_window_of_everything_is_the_causal_mask(dtype, D):
    c = Chunk([(150, 200), (70, 0)], 4, 2, D, dtype, seed=3)
    got = c.run(HUGE, 0)
    fp = B.make_fwd_params(c.q, c.k, c.v, c.o, c.lse, c.cu_q, c.cu_k, c.scale)
    B.cf_attn_fwd(fp)
    torch.cuda.synchronize()
    # Both are within W.tolerances of the exact o: half a step of o each, and where P enters the second product rounded to bf16, 2^-8 of
    # sum P |v| (some kernels of either call do that, others keep 16 bits or more): so far apart, at most, are the two.
    ref = c.reference(10**6, 0)
    tol = W.tolerances(ref, dtype, D, dtype == BF16)["o"]
    assert bool(((got["o"].double() - c.o.double()).abs() <= 2 * tol).all())
    assert float((got["lse"] - c.lse).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_keys_that_nobody_sees_are_left_alone(dtype, D, flags):
    """Infinities and NaNs there change nothing, and their gradients stay as they were, bit for bit."""
    c = Chunk([(40, 600)], 4, 2, D, dtype, seed=5)
    ref = c.reference(100, 4)
    hidden = slice(4, 501)                           # 600 - 99 = 501 is the first key of the first row
    c.k[hidden], c.v[hidden] = float("nan"), float("inf")
    got = c.run(100, 4, flags)
    c.check(got, ref, "hidden keys")
    assert torch.equal(got["dk"][hidden], c.start[0][hidden]) and torch.equal(got["dv"][hidden], c.start[1][hidden])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_a_row_that_is_not_finite_reaches_those_that_see_it(dtype, D, flags, value):
    """One value of V (and of K) of key 70 of 200, window 50, no sinks: rows 70 .. 119 see it, no other row changes."""
    for which in ("v", "k"):
        c = Chunk([(200, 0)], 4, 2, D, dtype, seed=6)
        good = c.run(50, 0, flags | ONE)
        getattr(c, which)[70, 1, 5] = value
        got = c.run(50, 0, flags | ONE)
        rows = torch.ones(200, dtype=torch.bool, device=DEV)
        rows[70:120] = False
        for name in ("o", "dq"):
            assert torch.isfinite(got[name][rows]).all(), (which, name)
            # (rows whose block was taken again pair by pair: sums in another order)
            assert torch.allclose(got[name][rows].float(), good[name][rows].float(), atol=2.0 ** -6 if dtype == BF16 else 1e-5, rtol=0), (which, name)
        assert torch.isfinite(got["lse"][:, rows]).all()
        # keys that no poisoned row sees: a row 70 .. 119 sees keys 21 .. 119
        keys = torch.ones(200, dtype=torch.bool, device=DEV)
        keys[21:120] = False
        for name in ("dk", "dv"):
            assert torch.isfinite(got[name][keys]).all(), (which, name)
            assert torch.isfinite(got[name][:, 0]).all()         # the other key/value head
        if value != value and which == "k":
            assert torch.isnan(got["o"][70:120, 2:]).all() and torch.isfinite(got["o"][70:120, :2]).all()


@pytest.mark.parametrize("dtype,D,flags", KINDS)
def test_a_far_row_that_is_not_finite(dtype, D, flags):
    """One value of dO of the last of 700 rows, window 50, 3 sinks: the gradients of the keys it sees, the sinks among them, and of no other."""
    c = Chunk([(700, 0)], 4, 2, D, dtype, seed=12)
    c.d_o[699, 3, 7] = float("inf")
    got = c.run(50, 3, flags | ONE)
    assert torch.isfinite(got["dq"][:699]).all() and torch.isfinite(got["dv"][3:650]).all() and torch.isfinite(got["dk"][3:650]).all()
    assert torch.isfinite(got["dv"][:, 0]).all() and not torch.isfinite(got["dv"][:3, 1, 7]).any() and torch.isfinite(got["dv"][:3, 1, 8:]).all()
    assert not torch.isfinite(got["dv"][650:, 1, 7]).any()


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
@pytest.mark.parametrize("dtype,D", [(FP32, 64), (BF16, 128)])
def test_other_scales(dtype, D, scale):
    c = Chunk([(70, 100)], 4, 2, D, dtype, seed=7, scale=scale)
    got, ref = c.run(60, 3), c.reference(60, 3)
    c.check(got, ref, scale)


@pytest.mark.parametrize("dtype,D,flags", [(FP32, 64, 0), (BF16, 64, 0), (BF16, 128, 0), (BF16, 128, ONE), (BF16, 64, ONE)])
def test_runs_repeat(dtype, D, flags):
    c = Chunk([(700, 300), (560, 0)], 8, 2, D, dtype, seed=8)
    a, b = c.run(200, 4, flags), c.run(200, 4, flags)
    for name in a:
        if name in ("dk", "dv") and dtype == BF16 and not flags:
            assert torch.allclose(a[name], b[name], atol=1e-4)
        else:
            assert torch.equal(a[name], b[name]), name


def test_gradients_against_differences_of_the_forward():
    """fp32: the loss <o, d_o> along one direction of q, k and v each, against <gradient, direction>.  The difference quotient's own error:
    h^2 times a third derivative (1e-4 of it), and 1e-6 sqrt(n) / h of rounding."""
    c = Chunk([(90, 60)], 4, 2, 64, FP32, seed=9)
    got = c.run(40, 3)
    grads = dict(q=got["dq"], k=got["dk"] - c.start[0], v=got["dv"] - c.start[1])
    for name, grad in grads.items():
        x = getattr(c, name)
        u = torch.randn(x.shape, device=DEV)
        keep, loss = x.clone(), []
        for h in (1e-2, -1e-2):
            x.copy_(keep + h * u)
            loss.append(float((c.run(40, 3, backward=False)["o"].double() * c.d_o.double()).sum()))
        x.copy_(keep)
        want = float((grad.double() * u.double()).sum())
        assert abs((loss[0] - loss[1]) / 2e-2 - want) < 2e-3 * float(grad.double().norm() * 1.0), (name, loss, want)


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP32, 64)])
def test_other_streams_and_graphs(dtype, D):
    """A forward and a backward captured into a graph, replayed with eager work of the same buffers in between."""
    c = Chunk([(300, 100), (41, 0)], 4, 2, D, dtype, seed=11)
    want = c.run(70, 2, ONE)
    fp = B.make_fwd_params(c.q, c.k, c.v, c.o, c.lse, c.cu_q, c.cu_k, c.scale, ONE)
    dkv = c.start.clone()
    ws = torch.empty(B.cf_attn_window_bwd_workspace_bytes(fp, 70, 2), dtype=torch.uint8, device=DEV)
    bp = B.make_bwd_params(fp, c.d_o, c.dq, dkv[0], dkv[1], ws)

    def step():
        dkv.copy_(c.start)
        B.cf_attn_window_fwd(fp, 70, 2)
        B.cf_attn_window_bwd(bp, 70, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        for x in (c.o, c.lse, c.dq, dkv, ws):
            x.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, x in (("o", c.o), ("lse", c.lse), ("dq", c.dq), ("dk", dkv[0]), ("dv", dkv[1])):
            assert bool(torch.equal(x, want[name])), (replay, name)
