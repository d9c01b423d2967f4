"""CPU checks of the pages that a window gives back: which ones, and that a call looks at the new ones only, however long the sequence is."""
import random

import pytest
import torch

from paper_2503_02356_amd.paged import PagedCache


@pytest.fixture(autouse=True)
def bookkeeping_only(monkeypatch):
    monkeypatch.setattr(PagedCache, "_append_and_attend", lambda self, names, counts, q, k, v, scale, lse: torch.zeros_like(q))


def attend(cache, name, n):
    q = torch.zeros(n, 1, 64, dtype=torch.bfloat16)
    cache.attend([name], [n], q, q, q)


@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (16, 4), (33, 16), (40, 17), (7, 100)])
def test_pages_that_no_later_query_sees_are_free(page, window, sinks):
    rng = random.Random(window)
    cache = PagedCache(400, page, 1, 64, device="cpu", window=window, n_sinks=sinks)
    length = {"a": 0, "b": 0}
    for step in range(60):
        name = rng.choice("ab")
        n = rng.choice([1, 1, 1, 2, 9, 40])
        attend(cache, name, n)
        length[name] += n
        held = []
        for name in cache.seqs:
            total, pages = cache.seqs[name]
            assert total == length[name] and len(pages) == -(-total // page)
            # key j is seen by the next token, at position total, or a later one iff j > total - window or j < sinks
            # (and the rest of the last page is for tokens to come)
            want = [any(j > total - window or j < sinks for j in range(c * page, min((c + 1) * page, total))) or (c + 1) * page > total - window + 1
                    for c in range(len(pages))]
            assert [p >= 0 for p in pages] == want, (step, name)
            held += [p for p in pages if p >= 0]
        assert sorted(held + cache.free) == list(range(400))


class Watched(list):
    looked = 0

    def __getitem__(self, i):
        Watched.looked += 1
        return list.__getitem__(self, i)


def test_a_long_sequence_is_not_gone_through():
    cache = PagedCache(300, 16, 1, 64, device="cpu", window=100, n_sinks=20)
    attend(cache, "a", 1)
    for _ in range(400):
        attend(cache, "a", 64)                       # 1600 columns, some 10 pages
    assert cache.used_pages() < 20
    cache.seqs["a"][1] = Watched(cache.seqs["a"][1])
    Watched.looked = 0
    for _ in range(32):
        attend(cache, "a", 1)
    assert Watched.looked < 32 * 8, Watched.looked
