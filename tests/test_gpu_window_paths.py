"""The runner, the executor and the paged cache with windows and sinks: whole plans against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2503_02356_amd import binding as B
from paper_2503_02356_amd import inputs
from paper_2503_02356_amd.executor import SlotExecutor
from paper_2503_02356_amd.paged import PagedCache, plan_forward
from paper_2503_02356_amd.runner import ChunkAttention
from tests import parity as P
from tests import plain_window as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LENS, C = [900, 40, 300, 1500, 77, 256, 1, 129], 256


def definition(lens, Hq, Hkv, D, dtype, seed, window, sinks):
    out = {}
    for sid, L in enumerate(lens):
        s = {n: torch.from_numpy(np.asarray(x, dtype=np.float64)).to(DEV) for n, x in inputs.seq_values(seed, sid, L, Hq, Hkv, D, dtype).items()}
        r = W.chunk(s["q"], s["k"], s["v"], float(np.float32(1 / np.sqrt(D))), [(L, 0)], window, sinks, s["d_o"])
        out[sid] = {n: r[n].cpu().numpy() for n in P.NAMES}
    return out


@pytest.mark.parametrize("dtype,D,window,sinks,kw", [
    ("bf16", 128, 100, 4, {}), ("bf16", 64, 300, 0, {}), ("fp32", 64, 37, 16, {}), ("bf16", 128, 100, 4, dict(K=1)),
    ("bf16", 128, 400, 2, dict(n_streams=2)), ("bf16", 128, 100, 4, dict(merge=True)), ("bf16", 128, 100, 4, dict(graph=True)),
    ("fp32", 128, 100, 4, dict(graph=True))])
def test_runner(dtype, D, window, sinks, kw):
    plan = B.cf_build_chunks_ex(LENS, C, B.CF_PLAN_MERGE_TAILS) if kw.get("merge") else B.cf_build_chunks(LENS, C)
    vals = lambda sid, L: inputs.seq_values(5, sid, LENS[sid], 4, 2, D, dtype)
    eng = ChunkAttention(plan, 4, 2, D, dtype, window=window, n_sinks=sinks, n_streams=kw.get("n_streams", 1)).load(vals)
    ref = definition(LENS, 4, 2, D, dtype, 5, window, sinks)
    want = sum(int(W.visible(L, L, window, sinks).sum()) for L in LENS)
    assert eng.total_pairs == want
    if kw.get("graph"):
        graph = eng.capture_step()
        for _ in range(3):
            for ch in eng.chunks:
                ch["o"].fill_(7), ch["d_q"].fill_(7), ch["lse"].fill_(7)
            eng.grad_arena.fill_(3)
            torch.cuda.synchronize()
            graph.replay()
            P.check(eng.results(), ref, dtype, "replay")
        return
    if kw.get("K"):
        eng.run_schedule(kw["K"])
    else:
        eng.run_forward()
        eng.run_backward()
    P.check(eng.results(), ref, dtype, (window, sinks, kw))


def test_runner_refuses_a_window_with_fused_launches():
    plan = B.cf_build_chunks([10], 16)
    with pytest.raises(ValueError, match="fused"):
        ChunkAttention(plan, 2, 1, 64, "bf16", window=4, fused_launch=True)


@pytest.mark.parametrize("K,dtype,D", [(1, "bf16", 128), (3, "fp32", 64)])
def test_executor(K, dtype, D):
    plan = B.cf_build_chunks(LENS, C)
    ex = SlotExecutor(plan, 4, 2, D, dtype, K, window=120, n_sinks=3).load(lambda sid, L: inputs.seq_values(6, sid, LENS[sid], 4, 2, D, dtype))
    ex.run()
    P.check(ex.results(), definition(LENS, 4, 2, D, dtype, 6, 120, 3), dtype, K)


@pytest.mark.parametrize("dtype,D,window,sinks,merge", [("bf16", 128, 0, 0, False), ("bf16", 128, 100, 4, False), ("bf16", 64, 100, 20, True),
                                                        ("fp32", 64, 70, 1, True)])
def test_plan_over_a_paged_cache(dtype, D, window, sinks, merge):
    """Append and attention of every chunk in turn: O and LSE of whole plans; with a window a sequence of 1500 tokens holds no more pages
    than a chunk, a window and the sinks need."""
    plan = B.cf_build_chunks_ex(LENS, C, B.CF_PLAN_MERGE_TAILS) if merge else B.cf_build_chunks(LENS, C)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    vals = {sid: inputs.seq_values(7, sid, L, 4, 2, D, dtype) for sid, L in enumerate(LENS)}
    cache = PagedCache(120, 16, 2, D, tdt, DEV, window, sinks)
    for x in (cache.k_pages, cache.v_pages):
        x.fill_(float("nan"))                        # (what a program never wrote)

    def rows(c):
        cat = lambda n: torch.from_numpy(np.concatenate([vals[sid][n][a:a + m] for sid, a, m in plan.chunk_segments(c)])).to(DEV).to(tdt)
        return cat("q"), cat("k"), cat("v")
    got = {sid: dict(o=np.zeros((L, 4, D)), lse=np.zeros((4, L))) for sid, L in enumerate(LENS)}
    for c, o, lse in plan_forward(plan, cache, rows, float(np.float32(1 / np.sqrt(D)))):
        row = 0
        for sid, a, n in plan.chunk_segments(c):
            got[sid]["o"][a:a + n] = o[row:row + n].double().cpu().numpy()
            got[sid]["lse"][:, a:a + n] = lse[:, row:row + n].double().cpu().numpy()
            row += n
    ref = definition(LENS, 4, 2, D, dtype, 7, window, sinks)
    P_names, P.NAMES = P.NAMES, ("o", "lse")
    try:
        P.check(got, ref, dtype, (window, sinks, merge))
    finally:
        P.NAMES = P_names
    assert cache.used_pages() == 0 and not cache.seqs
    if window and not merge:
        assert cache.peak_pages <= -(-(C + window + 16) // 16) + 1 + -(-sinks // 16) < 1500 // 16


def test_tokens_one_by_one_equal_a_chunk():
    """A prompt as one chunk, then tokens one at a time beside another sequence that begins later, against the whole sequences at once."""
    Hq, Hkv, D, lens = 8, 2, 128, [60, 25]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    seqs = [tuple(torch.randn(n, H, D, generator=g, device=DEV).bfloat16() for H in (Hq, Hkv, Hkv)) for n in lens]
    cache = PagedCache(40, 16, Hkv, D, window=33, n_sinks=2)
    outs = [[], []]
    outs[0].append(cache.attend(["a"], [40], *(x[:40] for x in seqs[0])))
    for t in range(20):
        names, rows = ["a"], [tuple(x[40 + t:41 + t] for x in seqs[0])]
        if t >= 3:
            m = 9 if t == 3 else 1
            b = 0 if t == 3 else 5 + t
            names.append("b"), rows.append(tuple(x[b:b + m] for x in seqs[1]))
        o = cache.attend(names, [len(r[0]) for r in rows], *(torch.cat([r[i] for r in rows]) for i in range(3)))
        outs[0].append(o[:1])
        if t >= 3:
            outs[1].append(o[1:])
    for i, (q, k, v) in enumerate(seqs):
        ref = W.chunk(q, k, v, D ** -0.5, [(lens[i], 0)], 33, 2)
        o = torch.cat(outs[i])
        tol = W.tolerances(ref, torch.bfloat16, D, True)
        W.check(dict(o=o), ref, dict(o=tol["o"][:len(o)]) if len(o) == lens[i] else {}, i)
        assert len(o) == lens[i]
    with pytest.raises(MemoryError):
        cache.attend(["c"], [700], *(x.repeat(20, 1, 1)[:700] for x in seqs[0]))
    assert "c" not in cache.seqs
