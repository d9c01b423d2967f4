"""How many bits of P and dS reach the results: where the products take them whole, errors are those of the results' own type."""
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_window as W
from tests.test_gpu_paged import Batch
from tests.test_gpu_window import HUGE, Chunk

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("flags", [0, B.CF_FLAG_DKV_SINGLE_WRITER])
@pytest.mark.parametrize("segs,window,sinks,names", [([(100, 0)] * 8, HUGE, 0, ("dk", "dv")), ([(100, 0)] * 8, 60, 4, ("dk", "dv")),
                                                     ([(700, 900), (90, 0)], 60, 4, ("dk", "dv")), ([(700, 900), (90, 0)], 300, 4, ("dv",)),
                                                     ([(700, 900), (90, 0)], HUGE, 0, ("dv",))])
def test_windowed_gradients_at_head_dim_64(segs, window, sinks, names, flags):
    """dK and dV leave in fp32 and have P's and dS's 24 bits, as in the causal call: some 20 roundings of 2^-24 in a row, 1.2e-6 in the 2-norm at
    most.  (dK only where delta comes from P and dP, rows of up to 128 keys: the others' from an o that is rounded to bf16.)"""
    c = Chunk(segs, 8, 2, 64, BF16, seed=4)
    c.start.zero_()
    got, ref = c.run(window, sinks, flags), c.reference(min(window, 10**6), sinks)
    for name in names:
        off = float((got[name].double() - ref[name]).norm() / ref[name].norm())
        print(name, off)
        assert off < 20 * 2.0 ** -24, (name, off)


def check_rounding_of_o_alone(b, got, rows, what):
    """o is off by its own rounding and by what two bf16 operands leave of P: half a step of half a step, 2^-16 of sum P |v|."""
    ref = b.reference()
    tol = W.tolerances(ref, BF16, b.D, False)["o"] + 2.0 ** -16 * ref["o_abs"]
    W.check(dict(o=got["o"][rows]), dict(o=ref["o"][rows]), dict(o=tol[rows]), what)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 20)])
@pytest.mark.parametrize("page", [16, 64])
def test_paged_tiles_of_few_rows(D, page, window, sinks):
    b = Batch([(1, 5000), (2, 300), (1, 64), (8, 700)], 8, 2, D, BF16, page, window, sinks, seed=40)
    check_rounding_of_o_alone(b, b.run(max_kv_len=5000), slice(0, 12), "tokens")
    b = Batch([(1, 2000)] * 6 + [(300, 900)], 8, 2, D, BF16, page, window, sinks, seed=41)
    check_rounding_of_o_alone(b, b.run(), slice(0, 6), "tokens beside a chunk")


@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 20)])
@pytest.mark.parametrize("page", [16, 64])
def test_paged_tiles_of_many_rows_at_head_dim_64(page, window, sinks):
    """As cf_attn_fwd, which takes P whole there."""
    for seqs in ([(700, 1500)], [(1, 2000)] * 6 + [(300, 900)], [(40, 3000)], [(1, 60), (400, 400), (130, 900)]):
        b = Batch(seqs, 8, 2, 64, BF16, page, window, sinks, seed=42)
        check_rounding_of_o_alone(b, b.run(), slice(None), seqs)
