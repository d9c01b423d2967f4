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


def laid_out(how, q):
    """q of another layout."""
    T, Hq, D = q.shape
    if how == "expanded over tokens":
        return q[:1].expand(T, Hq, D)
    if how == "expanded over heads":
        return q[:, :1].expand(T, Hq, D)
    if how == "rows that overlap":
        return torch.as_strided(q, (T, Hq, D), (D // 2, D, 1))
    if how == "offset":
        return torch.zeros(T * Hq * D + 1, dtype=q.dtype)[1:].view(T, Hq, D)
    if how == "stride":
        return torch.zeros(T, Hq, D + 1, dtype=q.dtype)[:, :, :D]
    if how == "heads first":
        return torch.zeros(Hq, T, D, dtype=q.dtype).transpose(0, 1)
    if how == "a part of a projection":
        return torch.zeros(T, Hq + 4, D, dtype=q.dtype)[:, :Hq]
    return q


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("how,scale,lse,fine", [
    ("as it is", None, True, True), ("as it is", 3.402e38, False, True), ("as it is", -0.5, False, True), ("heads first", None, False, True),
    ("a part of a projection", None, True, True), ("expanded over tokens", None, False, False), ("expanded over heads", None, True, False),
    ("rows that overlap", None, False, False), ("offset", None, False, False), ("stride", None, False, False), ("as it is", float("nan"), True, False),
    ("as it is", -float("inf"), False, False), ("as it is", 1e39, False, False)])
def test_nothing_is_appended_that_the_attention_refuses(how, scale, lse, fine, dtype, monkeypatch):
    """As far as the launches, which a list takes the place of: both calls are made, or neither is.  And whether they are is what the entry point's own
    checks say of the same call (given a workspace that is too small, so that it ends there)."""
    from paper_2503_02356_amd import binding as B
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    called, made = [], []
    make = B.make_paged8_params
    monkeypatch.setattr(B, "make_paged8_params", lambda *a, **k: made.append(make(*a, **k)) or made[-1])
    monkeypatch.setattr(B, "cf_kv_append8", lambda p, turn: called.append("append"))
    monkeypatch.setattr(B, "cf_attn_paged8_fwd", lambda p: called.append("attend"))
    cache = PagedCache(10, 16, 2, 64, dtype=dtype, device="cpu", eight_bits=True)
    k = torch.zeros(8, 2, 64, dtype=dtype)
    q = laid_out(how, torch.zeros(8, 4, 64, dtype=dtype))
    attend = lambda: cache.attend(["a"], [8], q, k, k, scale=scale, lse=torch.zeros(4, 8) if lse else None)
    if fine:
        attend()
        assert called == ["append", "attend"] and cache.lengths() == {"a": 8}
    else:
        with pytest.raises(ValueError):
            attend()
        assert called == [] and state(cache) == state(PagedCache(10, 16, 2, 64, device="cpu"))
    p = made[-1]
    p.a.max_kv_len, p.a.pages_per_seq, p.a.table_stride = 0, 512, 512        # (so long that it is cut into parts)
    p.a.workspace, p.a.workspace_bytes = 256, 0
    assert B.cf_attn_paged8_workspace_bytes(p) > 0
    code = B.lib().cf_attn_paged8_fwd(p, None)
    assert code == B.CF_EINVAL and ("workspace has 0 bytes" in B.lib().cf_last_error().decode()) == fine
