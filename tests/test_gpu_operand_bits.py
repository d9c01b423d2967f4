"""How many bits of P and dS reach the results: where the products take them whole, errors are those of the results' own type."""
import pytest
import torch

from paper_2503_02356_amd import binding as B
from tests import plain_window as W
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
