"""CPU checks of a paged cache of 8 bits or one that rotates: what a call that is refused leaves behind."""
import pytest
import torch

from paper_2503_02356_amd.paged import PagedCache
from tests.test_paged_cache import state


@pytest.mark.parametrize("names,counts,error", [(["a"], [40], AssertionError),              # (tensors that are not on a GPU)
                                                (["a", "b"], [17, 30], AssertionError), (["a"], [200], MemoryError), (["a", "a"], [1, 1], ValueError)])
def test_a_refused_call_leaves_the_sequences_as_they_were(names, counts, error):
    cache = PagedCache(10, 16, 2, 64, device="cpu", eight_bits=True)
    assert cache.k_pages.dtype == torch.float8_e4m3fn and tuple(cache.v_scales.shape) == (10, 2, 1)
    cache.seqs["a"] = [20, [cache.free.pop(), cache.free.pop()]]
    before = state(cache)
    q, k = torch.zeros(210, 4, 64, dtype=torch.bfloat16), torch.zeros(210, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(error):
        cache.attend(names, counts, q, k, k)
    assert state(cache) == before


@pytest.mark.parametrize("change", [dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e39), dict(q="offset"), dict(q="stride"), dict(q="dtype")])
def test_what_the_attention_would_refuse_comes_before_the_append(change, monkeypatch):
    from paper_2503_02356_amd import binding as B
    called = []
    monkeypatch.setattr(B, "cf_kv_append8", lambda *a: called.append(a))
    cache = PagedCache(10, 16, 2, 64, device="cpu", eight_bits=True)
    q, k = torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    if change.get("q") == "offset":
        q = torch.zeros(8 * 256 + 1, dtype=torch.bfloat16)[1:].view(8, 4, 64)
    elif change.get("q") == "stride":
        q = torch.zeros(8, 4, 65, dtype=torch.bfloat16)[:, :, :64]
    elif change.get("q") == "dtype":
        q = q.float()
    with pytest.raises((ValueError, AssertionError)):
        cache.attend(["a"], [8], q, k, k, scale=change.get("scale"))
    assert not called and state(cache) == state(PagedCache(10, 16, 2, 64, device="cpu"))


def test_pages_hold_whole_blocks():
    with pytest.raises(ValueError):
        PagedCache(10, 24, 2, 64, device="cpu", eight_bits=True)
