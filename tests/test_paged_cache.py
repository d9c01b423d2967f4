"""CPU checks of the paged cache's bookkeeping: what a call that is refused leaves behind."""
import pytest
import torch

from paper_2503_02356_amd.paged import PagedCache


def state(cache):
    return list(cache.free), {name: (n, list(pages)) for name, (n, pages) in cache.seqs.items()}


@pytest.mark.parametrize("names,counts,error", [(["a"], [40], AssertionError),              # (tensors that are not on a GPU)
                                                (["a", "b"], [17, 30], AssertionError), (["b", "c"], [1, 1], AssertionError),
                                                (["a"], [200], MemoryError), (["a", "a"], [1, 1], ValueError), (["a"], [-1], ValueError),
                                                (["a", "b"], [1], ValueError), (["a"], [1, 1], ValueError), ([], [], ValueError)])
def test_a_refused_call_leaves_the_sequences_as_they_were(names, counts, error):
    cache = PagedCache(10, 16, 2, 64, device="cpu")
    cache.seqs["a"] = [20, [cache.free.pop(), cache.free.pop()]]
    before = state(cache)
    q, k = torch.zeros(210, 4, 64, dtype=torch.bfloat16), torch.zeros(210, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(error):
        cache.attend(names, counts, q, k, k)
    assert state(cache) == before
