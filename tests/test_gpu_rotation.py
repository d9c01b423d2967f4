"""Rotation of a chunk's queries and keys, their gradients, and the append that rotates on the way, against the definition in 64 bits."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_cache8 as P
from tests.test_gpu_paged import Batch, ints

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1234)


def frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(rot // 2, device=DEV, dtype=torch.float64) / (rot // 2))).float()


def positions(segs):
    return torch.cat([torch.arange(lk - lq, lk, device=DEV) for lq, lk in segs])


def lists(segs):
    return ints(np.cumsum([0] + [a for a, _ in segs])), ints(np.cumsum([0] + [b for _, b in segs]))


def close(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (what, float((off - tol).max()), (off > tol).nonzero()[:4].tolist())


SEGS = [[(1, 1)], [(1, 2**30)], [(333, 1333)], [(3, 3), (70, 70), (1, 1), (64, 64), (200, 200)], [(5, 1 << 20), (40, 229376 + 40)], [(1, 1)] * 300 + [(7, 7)]]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (128, 112), (128, 16), (64, 64), (64, 48)])
@pytest.mark.parametrize("s", range(len(SEGS)))
def test_there_and_back(s, D, rot, interleaved):
    """q in bf16 and k in fp32 there; dQ in bf16 and dK from fp32 to bf16 back.  Rows behind the last segment stay."""
    segs, f, pad, Hq, Hkv = SEGS[s], frequencies(rot), s % 3, [7, 32, 5][s % 3], [1, 4, 2][s % 3]
    T, pos = sum(a for a, _ in segs), positions(segs)
    g = torch.Generator(device=DEV)
    g.manual_seed(s)
    rnd = lambda H, dt: torch.randn(T + pad, H, D, generator=g, device=DEV).to(dt)
    cu_q, cu_k = lists(segs)
    qkv = rnd(Hq + 2 * Hkv, BF16)
    r = B.make_rotation(f, interleaved)
    for q, k, to, back in ((qkv[:, :Hq], rnd(Hkv, FP32), FP32, False), (rnd(Hq, BF16), rnd(Hkv, FP32), BF16, True)):
        yq, yk = torch.full_like(q, 7.0), torch.full((T + pad, Hkv, D), 7.0, device=DEV, dtype=to)
        B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, q=(q, yq), k=(k, yk), inverse=back))
        torch.cuda.synchronize()
        for x, y in ((q, yq), (k, yk)):
            want, tol = P.turn_tolerance(x[:T], pos, f, interleaved, back, y.dtype)
            close(y[:T], want, tol, (segs[:3], D, rot, back))
            assert bool((y[T:] == 7.0).all())
            assert bool(torch.equal(y[:T, :, rot:], x[:T, :, rot:].to(y.dtype)))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [(BF16, 128, 128), (FP32, 64, 32), (BF16, 64, 64), (FP32, 128, 96)])
def test_in_place_and_one_tensor(dtype, D, rot, interleaved):
    segs = [(50, 90), (131, 131)]
    cu_q, cu_k = lists(segs)
    f = frequencies(rot, 500000.0)
    r = B.make_rotation(f, interleaved)
    buffer = torch.randn(181, 9, D, device=DEV).to(dtype)
    q, keep = buffer[:, 2:8], buffer.clone()
    want, tol = P.turn_tolerance(q, positions(segs), f, interleaved, False, dtype)
    B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, q=(q, q)))
    torch.cuda.synchronize()
    close(q, want, tol, "in place")
    assert bool(torch.equal(buffer[:, :2], keep[:, :2])) and bool(torch.equal(buffer[:, 8:], keep[:, 8:]))
    heads_first = torch.empty(9, 181, D, device=DEV, dtype=dtype).transpose(0, 1)
    B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, k=(keep, heads_first)))
    torch.cuda.synchronize()
    assert bool(torch.equal(heads_first[:, 2:8], q))


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_gradient_is_that_of_the_formula(interleaved):
    """<R x, y> = <x, R' y> for any x, y; and against differences of a function of the rotated values."""
    segs, D = [(40, 640), (23, 23)], 64
    cu_q, cu_k = lists(segs)
    r = B.make_rotation(frequencies(D), interleaved)
    x, w = (torch.randn(63, 3, D, device=DEV) for _ in range(2))
    turn = lambda a, back=False: (lambda y: (B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, q=(a, y), inverse=back)), y)[1])(torch.empty_like(a))
    y = turn(x)
    grad = turn(torch.cos(y) * w, True)              # of sum w sin(R x)
    plain = x.double().requires_grad_()
    (torch.sin(P.turned(plain, positions(segs), frequencies(D), interleaved)[0]) * w).sum().backward()
    assert float((grad - plain.grad).abs().max()) < 64 * 2.0 ** -24 * 5
    step, at = 2.0 ** -8, (50, 1, 5)
    up, down = x.clone(), x.clone()
    up[at] += step
    down[at] -= step
    loss = lambda a: float((torch.sin(turn(a).double()) * w).sum())
    # the third derivative of sum w sin(R x) along one element is at most sum |w| over a pair; fp32 results of 12096 terms
    assert abs((loss(up) - loss(down)) / (2 * step) - float(grad[at])) < 10 * step ** 2 + 2.0 ** -24 * 12 / step


def test_what_is_not_finite_stays_in_its_pair():
    cu_q, cu_k = lists([(6, 6)])
    for interleaved in (False, True):
        x = torch.randn(6, 2, 128, device=DEV)
        x[3, 1, 10] = float("inf")
        y = torch.empty_like(x)
        B.cf_rotate(B.make_rotate_params(cu_q, cu_k, B.make_rotation(frequencies(64), interleaved), q=(x, y)))
        torch.cuda.synchronize()
        bad = (~torch.isfinite(y)).nonzero().tolist()
        other = 11 if interleaved else 42
        assert bad == [[3, 1, 10], [3, 1, other]]


def test_many_heads_and_rows():
    """Groups of heads that do not divide them; many rows; another stream."""
    segs = [(4097, 4097 + 100), (3000, 3000)]
    cu_q, cu_k = lists(segs)
    f = frequencies(128)
    q, k = torch.randn(7097, 71, 128, device=DEV).to(BF16), torch.randn(7097, 3, 128, device=DEV).to(BF16)
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.cf_rotate(B.make_rotate_params(cu_q, cu_k, B.make_rotation(f), q=(q, yq), k=(k, yk)))
    torch.cuda.current_stream().wait_stream(side)
    for x, y in ((q, yq), (k, yk)):
        want, tol = P.turn_tolerance(x, positions(segs), f, False, False, BF16)
        close(y, want, tol, "many")


@pytest.mark.parametrize("dtype,D,rot,interleaved", [(BF16, 128, 128, False), (BF16, 64, 32, True), (FP32, 128, 96, False), (FP32, 64, 64, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_rotated(dtype, D, rot, interleaved, in_place):
    """Across page ends, into the middle of a page, positions before the first, pages that are none, padded rows; queries by the way."""
    hidden = {(0, 2): -1, (3, 0): 10**9}
    b = Batch([(40, 50), (1, 16), (1, 17), (3, 9), (5, 2), (0, 30), (0, 0), (1, 5000)], 6, 2, D, dtype, 16, hidden=hidden, pad=3, seed=11)
    f = frequencies(rot)
    T, pos = 51, torch.cat([torch.arange(n - a, n, device=DEV) for a, n in b.seqs]).clamp(min=0)
    for x in (b.kp, b.vp):
        x.copy_(torch.randn(x.shape, device=DEV).to(dtype))
    keep, q = [x.clone() for x in (b.kp, b.vp)], b.q.clone()
    q_out = b.q if in_place else torch.full_like(b.q, 7.0)
    call = lambda: B.cf_kv_append_rotated(B.make_kv_append_params(b.k, b.v, b.kp, b.vp, b.cu, b.lens, b.table),
                                          B.make_append_rotation(B.make_rotation(f, interleaved), b.q, q_out))
    call()
    torch.cuda.synchronize()
    want, tol = P.turn_tolerance(q[:T], pos, f, interleaved, False, dtype)
    close(q_out[:T], want, tol, "queries")
    assert bool(torch.equal(q_out[T:], q[T:] if in_place else torch.full_like(q[T:], 7.0)))
    want, tol = P.turn_tolerance(b.k[:T], pos, f, interleaved, False, dtype)
    written = torch.zeros(b.n_pages, 16, dtype=torch.bool, device=DEV)
    row = 0
    for i, (a, n) in enumerate(b.seqs):
        for r in range(a):
            j = n - a + r
            at = int(b.table_host[i, j // 16]) if j >= 0 else -1
            if 0 <= at < b.n_pages:
                written[at, j % 16] = True
                close(b.kp[at, j % 16], want[row + r], tol[row + r], ("key", i, r))
                assert bool(torch.equal(b.vp[at, j % 16], b.v[row + r]))
        row += a
    for x, old in zip((b.kp, b.vp), keep):
        assert bool(torch.equal(x[~written], old[~written])) and int(written.sum()) == 51 - 16 - 3 - 3


def test_append_rotated_without_queries_and_rotate_agree():
    """The cache holds what cf_rotate gives a training chunk at the same positions, bit by bit."""
    segs = [(100, 420), (33, 33)]
    b = Batch(segs, 4, 2, 128, BF16, 64, seed=3)
    f = frequencies(128)
    r = B.make_rotation(f)
    B.cf_kv_append_rotated(B.make_kv_append_params(b.k, b.v, b.kp, b.vp, b.cu, b.lens, b.table), B.make_append_rotation(r))
    y = torch.empty(b.k.shape, dtype=BF16, device=DEV)
    cu_q, cu_k = lists(segs)
    B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, k=(b.k, y)))
    torch.cuda.synchronize()
    row = 0
    for i, (a, n) in enumerate(segs):
        for r_ in range(a):
            j = n - a + r_
            assert bool(torch.equal(b.kp[int(b.table_host[i, j // 64]), j % 64], y[row + r_]))
        row += a


def test_graph_of_both():
    """A captured step of append and rotation, replayed with other rows and lengths."""
    b = Batch([(1, 700), (2, 33)], 4, 2, 64, FP32, 16, columns=1, seed=4)
    b.table_host[:, -1] = 1                          # (not reached)
    f = frequencies(64)
    q_out = torch.empty_like(b.q)
    p, t = B.make_kv_append_params(b.k, b.v, b.kp, b.vp, b.cu, b.lens, b.table), B.make_append_rotation(B.make_rotation(f), b.q, q_out)
    B.cf_kv_append_rotated(p, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cf_kv_append_rotated(p, t)
    for step in range(4):
        b.lens.copy_(ints([700 - step, 33 - 2 * step]))
        b.q.copy_(torch.randn(b.q.shape, device=DEV)), b.k.copy_(torch.randn(b.k.shape, device=DEV))
        q_out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        pos = torch.tensor([699 - step, 31 - 2 * step, 32 - 2 * step], device=DEV)
        for x, y in ((b.q, q_out), (b.k, torch.stack([b.kp[int(b.table_host[i, j // 16]), j % 16] for i, j in zip((0, 1, 1), pos.tolist())]))):
            want, tol = P.turn_tolerance(x, pos, f, False, False, FP32)
            close(y, want, tol, step)


@pytest.mark.parametrize("D,dtype,interleaved", [(128, BF16, False), (64, BF16, True), (128, FP32, False)])
def test_a_large_call_does_what_its_segments_calls_do(D, dtype, interleaved):
    """Several thousand rows, whose groups of heads and stores are others, against a call for each segment, bit by bit."""
    lens, pad = [3000, 1, 2500, 0, 70], 3
    T = sum(lens)
    q, k = torch.randn(T + pad, 14, D, device=DEV).to(dtype), torch.randn(T + pad, 3, D, device=DEV).to(dtype)
    rotation, cu = B.make_rotation(frequencies(D), interleaved), np.cumsum([0] + lens)
    cu_k = np.cumsum([0] + [n + 100 * (n > 1) for n in lens])
    ys = [[torch.full_like(x, 7.0) for x in (q, k)] for _ in range(2)]
    B.cf_rotate(B.make_rotate_params(ints(cu), ints(cu_k), rotation, (q, ys[0][0]), (k, ys[0][1])))
    for a, b, n in zip(cu[:-1], cu[1:], np.diff(cu_k)):
        if b > a:
            B.cf_rotate(B.make_rotate_params(ints([0, b - a]), ints([0, n]), rotation, (q[a:b], ys[1][0][a:b]), (k[a:b], ys[1][1][a:b])))
    torch.cuda.synchronize()
    for x, y in zip(*ys):
        assert bool(torch.equal(x, y)) and bool((x[T:] == 7.0).all())


PI = Fraction(3141592653589793238462643383279502884197169399375105820974944592, 10 ** 63)


def turned_exactly(x, pos, f, interleaved):
    """P.turned with whole turns taken from the angles as fractions, and the tolerance of fp32 results: a part of a turn rounded to fp32 (half a step of a number of
    half-turns, which may lie above 1: pi 2^-24), sine and cosine (2 steps of numbers up to 1: 2^-23), products and their sum (2^-24 each), fp64 besides."""
    angle = torch.tensor([[float((Fraction(w) * p / PI) % 2) * np.pi for w in f.tolist()] for p in pos.tolist()], dtype=torch.float64, device=DEV)
    rot = 2 * f.numel()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b, c, s = x[..., first].double(), x[..., second].double(), torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y, tol = x.double(), torch.zeros_like(x, dtype=torch.float64)
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    w = 3.15 * 2.0 ** -24 + 2.0 ** -23 + 2.0 ** -48
    for part, size in ((first, (a * c).abs() + (b * s).abs()), (second, (a * s).abs() + (b * c).abs())):
        tol[..., part] = w * (a.abs() + b.abs()) + 3 * 2.0 ** -24 * size
    return y, 1.001 * tol


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 64)])
@pytest.mark.parametrize("segs", [[(3, 2**31 - 1)], [(2, 2**30 + 1), (1, 229377), (1, 1)]])
def test_far_positions_are_as_exact_as_near_ones(segs, D, rot, interleaved):
    """Frequencies up to a turn a position and more: no part of the tolerance grows with the position.  And so are the keys and queries of an append."""
    f = frequencies(rot)
    f[:6] = torch.tensor([2 * np.pi, np.pi, 1.0, 100.0, -3.0, 1e-30], device=DEV)
    pos, (cu_q, cu_k), r = positions(segs), lists(segs), B.make_rotation(f, interleaved)
    x = torch.randn(int(cu_q[-1]), 2, D, device=DEV)
    y = torch.empty_like(x)
    B.cf_rotate(B.make_rotate_params(cu_q, cu_k, r, q=(x, y)))
    torch.cuda.synchronize()
    want, tol = turned_exactly(x, pos, f, interleaved)
    close(y, want, tol, (segs, D, interleaved))
    page, columns = 65536, 2**30 // 65536
    pos = torch.tensor([2**30 - 3, 2**30 - 2, 2**30 - 1], device=DEV)
    x = torch.randn(3, 4, D, device=DEV)
    table = torch.full((1, columns), -1, device=DEV, dtype=torch.int32)
    table[0, -1] = 0
    pages, q_out = torch.zeros(2, 1, page, 1, D, device=DEV), torch.empty(3, 2, D, device=DEV)
    append = B.make_kv_append_params(x[:, 2:3], x[:, 3:], pages[0], pages[1], ints([0, 3]), ints([2**30]), table)
    B.cf_kv_append_rotated(append, B.make_append_rotation(r, x[:, :2], q_out))
    torch.cuda.synchronize()
    for got, of in ((q_out, x[:, :2]), (pages[0, 0, -3:], x[:, 2:3])):
        want, tol = turned_exactly(of, pos, f, interleaved)
        close(got, want, tol, (D, interleaved))
    assert bool(torch.equal(pages[1, 0, -3:], x[:, 3:])) and not bool(pages[:, 0, :-3].any())
