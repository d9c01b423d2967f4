"""cf_kv_append where rows and sequences do not fill wavefronts: thousands of sequences, long runs of empty ones, a few rows in the last wavefront."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


NEW = {
    "one token each": [1] * 4201,
    "few rows behind many empty ones": [1] + [0] * 4000 + [1, 1],
    "rows between runs of empty ones": ([1] + [0] * 90) * 30 + [3] + [0] * 2000 + [2, 1],
    "all behind the empty ones": [0] * 5000 + [5],
    "before them": [5] + [0] * 5000,
    "one sequence": [7],
}


@pytest.mark.parametrize("dtype,Hkv,D", [(torch.bfloat16, 1, 64), (torch.bfloat16, 3, 128), (torch.float32, 2, 64)])
@pytest.mark.parametrize("name", NEW)
@pytest.mark.parametrize("pad", [0, 3])
def test_append_of_many_sequences(name, dtype, Hkv, D, pad):
    new, page = NEW[name], 16
    rng = np.random.default_rng(1)
    kept = rng.integers(0, 2 * page - 5, size=len(new))
    T, n_pages = sum(new), 2 * len(new)
    table = rng.permutation(n_pages).reshape(len(new), 2)
    k, v = (torch.randn(T + pad, Hkv, D, device=DEV).to(dtype) for _ in range(2))
    pages = [torch.zeros(n_pages, page, Hkv, D, device=DEV, dtype=dtype) for _ in range(2)]
    seq = np.repeat(np.arange(len(new)), new)
    at = kept[seq] + np.concatenate([np.arange(n) for n in new])
    where = table[seq, at // page] * page + at % page
    assert len(set(where.tolist())) == T and 0 <= where.min() and where.max() < n_pages * page
    want = [torch.zeros_like(p) for p in pages]
    for w, x in zip(want, (k, v)):
        w.view(-1, Hkv, D)[torch.tensor(where, device=DEV)] = x[:T]
    cu = ints(np.cumsum([0] + new))
    B.cf_kv_append(B.make_kv_append_params(k, v, *pages, cu, ints(kept + np.array(new)), ints(table)))
    torch.cuda.synchronize()
    for p, w in zip(pages, want):
        assert bool(torch.equal(p, w))
