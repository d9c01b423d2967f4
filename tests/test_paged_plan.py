"""CPU checks of what a plan's forward passes leave of a cache that others use: the bookkeeping runs, the calls of the library do not."""
import pytest
import torch

from paper_2503_02356_amd import binding as B
from paper_2503_02356_amd.paged import PagedCache, plan_forward

LENS, C = [40, 100, 3, 17], 32


def state(cache):
    return sorted(cache.free), {name: (n, list(pages)) for name, (n, pages) in cache.seqs.items()}


@pytest.fixture
def cache(monkeypatch):
    """A cache in which conversations 0, 1 and "a" are open: numbers that the plan's sequences have too."""
    monkeypatch.setattr(PagedCache, "_append_and_attend", lambda self, names, counts, q, k, v, scale, lse: torch.zeros_like(q))
    cache = PagedCache(40, 16, 1, 64, device="cpu")
    q, k = rows(70)
    cache.attend(["a", 0, 1], [20, 17, 33], q, k, k)
    return cache


def rows(n):
    return torch.zeros(n, 2, 64, dtype=torch.bfloat16), torch.zeros(n, 1, 64, dtype=torch.bfloat16)


def inputs_of(plan):
    def inputs(c):
        q, k = rows(sum(n for _, _, n in plan.chunk_segments(c)))
        return q, k, k
    return inputs


def test_other_sequences_stay(cache):
    plan, before = B.cf_build_chunks(LENS, C), state(cache)
    inputs = inputs_of(plan)
    chunks = []
    for c, o, lse in plan_forward(plan, cache, inputs):
        chunks.append(c)
        assert o.shape[0] == lse.shape[1] == sum(n for _, _, n in plan.chunk_segments(c))
        now = state(cache)[1]
        assert all(now[name] == s for name, s in before[1].items()) and len(now) > 3
        held = [p for _, pages in now.values() for p in pages]
        assert len(held) == len(set(held)) == cache.used_pages()
    assert sorted(chunks) == list(range(plan.n_chunks)) and state(cache) == before


def test_a_group_begins_with_no_keys(cache):
    """A sequence's slices find the tokens of its own earlier slices in the cache, and no others."""
    plan, seen = B.cf_build_chunks(LENS, C), {}

    def look(self, names, counts, q, *rest):
        seen[len(seen)] = [self.seqs[name][0] for name in names]
        return torch.zeros_like(q)
    cache._append_and_attend = look.__get__(cache)
    for n, (c, _, _) in enumerate(plan_forward(plan, cache, inputs_of(plan))):
        assert seen[n] == [a + m for _, a, m in plan.chunk_segments(c)]


def test_one_that_is_not_run_to_its_end_gives_its_pages_back(cache):
    plan, before = B.cf_build_chunks(LENS, C), state(cache)
    for stop in range(plan.n_chunks):
        passes = plan_forward(plan, cache, inputs_of(plan))
        for _ in range(stop + 1):
            next(passes)
        passes.close()
        assert state(cache) == before, stop


def test_a_cache_without_room(cache):
    plan = B.cf_build_chunks(LENS, C)
    q, k = rows(500)
    cache.attend(["b"], [16 * len(cache.free) - 40], q, k, k)
    before = state(cache)
    with pytest.raises(MemoryError):
        list(plan_forward(plan, cache, inputs_of(plan)))
    assert state(cache) == before


def test_two_at_once(cache):
    plan, before = B.cf_build_chunks(LENS, C), state(cache)
    passes = [plan_forward(plan, cache, inputs_of(plan)) for _ in range(2)]
    order = [(c, d) for (c, _, _), (d, _, _) in zip(*passes)]
    assert [c for c, _ in order] == [d for _, d in order] and len(order) == plan.n_chunks
    for p in passes:
        p.close()
    assert state(cache) == before
