"""The work of the windowed and of the paged attention calls, as a training and as a serving program makes them.

Kinds of a case
  fwd    one windowed forward call on one chunk: packed sequences, or a slice of one sequence behind the state of its earlier slices.
  step   that, and the backward call: key/value gradients cleared, accumulated in 32 bits (as over the slices of a sequence), and
         handed to the layers before in the model's type.
  serve  new tokens of a batch of sequences: their keys and values go into the pages of the cache (append), then they attend to all of it
         or to a window of it.  One token per sequence, chunks of a prompt, or both.

A query at position p of its sequence sees the keys j <= p with j > p - window (window 0: all) or j < sinks.
Sequence lengths are drawn from the case alone (lens_seed), values N(0, 1) from the seed that prepare() is given.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _chunk(name, kind, dtype, Hq, Hkv, D, T, prefix, median, window, sinks, packed=False, lens_seed=0):
    """median > 0: T tokens of packed sequences, lognormal (sigma 0.9) around it; 0: one slice of T tokens behind `prefix` keys.
    packed: q, k, v are views of one buffer, as one projection leaves them."""
    c = dict(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, T=T, prefix=prefix, median=median, window=window, sinks=sinks, packed=packed,
             lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def _serve(name, dtype, Hq, Hkv, D, page, n_tokens, n_chunks, chunk, least, most, window, sinks, append, lens_seed=0):
    """n_tokens sequences with one new token, n_chunks with `chunk` new tokens (each, a little fewer in every other one), behind `least` to
    `most` cached tokens, in pages of `page` tokens.  append: the new keys and values are written into the pages first."""
    c = dict(kind="serve", dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, page=page, n_tokens=n_tokens, n_chunks=n_chunks, chunk=chunk, least=least, most=most,
             window=window, sinks=sinks, append=append, lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a short last slice, evaluated: one small call, latency
        _chunk("tail_slice_fwd", "fwd", "bf16", 28, 4, 128, 33, 500, 0, 256, 4),
        # a layer checked in full precision
        _chunk("fp32_step", "step", "fp32", 6, 2, 128, 1000, 300, 0, 200, 2),
        # 64-wide heads, many short sequences, a window shorter than some of them
        _chunk("d64_packed_step", "step", "bf16", 16, 4, 64, 4096, 0, 300, 128, 4, packed=True),
        # a packed chunk of the 8K configuration
        _chunk("packed_8k_step", "step", "bf16", 28, 4, 128, 8192, 0, 600, 512, 4),
        # its longest sequence's last slice
        _chunk("slice_32k_step", "step", "bf16", 28, 4, 128, 8192, 24576, 0, 4096, 4),
        # the last slice of the 256K configuration, forward
        _chunk("slice_256k_fwd", "fwd", "bf16", 64, 8, 128, 32768, 229376, 0, 8192, 16),
        # one conversation, one token
        _serve("token_1", "bf16", 28, 4, 128, 16, 1, 0, 0, 4097, 4097, 0, 0, True),
        # a batch of conversations of different lengths
        _serve("tokens_64", "bf16", 32, 8, 128, 64, 64, 0, 0, 500, 16384, 0, 0, False),
        # a large batch of a model with windowed layers: pages behind the window have been given back
        _serve("tokens_256_window", "bf16", 16, 4, 64, 32, 256, 0, 0, 100, 20000, 1024, 4, True),
        # a chunk of a long prompt
        _serve("prompt_32k", "bf16", 28, 4, 128, 64, 0, 1, 8192, 24576, 24576, 0, 0, True),
        # a chunk of a prompt beside the single tokens of others
        _serve("mixed_41", "bf16", 32, 8, 128, 128, 40, 1, 500, 700, 9000, 0, 0, True),
        # the serving path checked in full precision
        _serve("fp32_serve", "fp32", 6, 2, 128, 16, 3, 2, 100, 20, 700, 0, 0, True),
    ]


_HEADS = [(28, 4), (32, 8), (64, 8), (16, 2), (8, 2), (4, 4), (14, 2), (16, 16)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: at most the arithmetic of slice_256k_fwd, a cache of 2 GB."""
    seed = rng.randrange(1, 1 << 30)
    kind = rng.choice(["fwd", "step", "step", "tokens", "tokens", "prompt", "mixed"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        D = rng.choice([64, 128, 128])
        Hq, Hkv = rng.choice(_HEADS) if dtype == "bf16" else rng.choice([(1, 1), (4, 4), (6, 2), (8, 2)])
        sinks = rng.choice([0, 1, 4, 4, 16, 64, 200])
        if kind in ("fwd", "step"):
            T = _log(rng, 1, 16384 if dtype == "bf16" else 2000)
            median = rng.choice([0, 0, _log(rng, 20, 2000)])
            prefix = 0 if median else rng.choice([0, _log(rng, 1, 100000 if dtype == "bf16" else 5000)])
            c = _chunk("", kind, dtype, Hq, Hkv, D, T, prefix, median, _log(rng, 1, 8192), sinks, rng.random() < 0.3 and prefix == 0, seed)
        else:
            one = 0 if kind == "prompt" else _log(rng, 1, 256)
            chunks = 0 if kind == "tokens" else rng.randint(1, 3)
            most = _log(rng, 1, 60000 if dtype == "bf16" else 5000)
            window = rng.choice([0, 0, _log(rng, 1, 8192)])
            c = _serve("", dtype, Hq, Hkv, D, rng.choice([16, 32, 64, 128, 256]), one, chunks, _log(rng, 2, 4096 if dtype == "bf16" else 300),
                       max(0, int(most * rng.random())), most, window, sinks if window else 0, rng.random() < 0.6, seed)
            new, kept = _lengths(c)
            if sum(new) + sum(kept) > (2 << 30) // (Hkv * D * 4 * (2 if dtype == "fp32" else 1)):
                continue
        new, kept = _lengths(c)
        widest = max(a + b for a, b in zip(new, kept))
        widest = min(widest, c["window"] + 400) if c["window"] else widest
        rows = sum(-(-n // _block_rows(c)) for n in new) * _block_rows(c)
        w = work(c)
        flop_most = (8e12 if dtype == "bf16" else 2e11)
        if w["flops"] <= flop_most and rows * (Hq // Hkv) * widest * 4 <= 6 << 30:
            return c


def _lengths(case):
    """(new tokens, tokens before them) of each sequence."""
    rng = random.Random(case["lens_seed"] * 7919 + 13)
    if case["kind"] == "serve":
        new = [1] * case["n_tokens"] + [max(1, case["chunk"] - (37 * (i % 2) if case["chunk"] > 64 else 0)) for i in range(case["n_chunks"])]
        kept = [rng.randint(case["least"], max(case["least"], case["most"])) for _ in new]
        return new, kept
    if case["median"] == 0:
        return [case["T"]], [case["prefix"]]
    new, left = [], case["T"]
    while left > 0:
        n = min(left, max(1, int(round(math.exp(rng.gauss(math.log(case["median"]), 0.9))))))
        new.append(n)
        left -= n
    return new, [0] * len(new)


def _block_rows(case):
    """Rows that the plain form takes together."""
    return 1 if case["kind"] == "serve" and case["n_chunks"] == 0 else 32 if case["kind"] == "serve" and case["n_tokens"] > 0 else 128


def _pairs(case):
    new, kept = _lengths(case)
    n = np.concatenate([np.arange(b + 1, a + b + 1) for a, b in zip(new, kept)]).astype(np.int64)     # keys up to its own
    if case["window"] == 0:
        return int(n.sum())
    beyond = np.maximum(n - case["window"], 0)
    return int((n - beyond + np.minimum(beyond, case["sinks"])).sum())


def _rows_read(case):
    """Key rows that some query sees."""
    new, kept = _lengths(case)
    rows = 0
    for a, b in zip(new, kept):
        first = max(0, b + 1 - case["window"]) if case["window"] else 0
        rows += a + b - first + min(first, case["sinks"])
    return rows


def work(case):
    new, _ = _lengths(case)
    size = 2 if case["dtype"] == "bf16" else 4
    q, kv = sum(new) * case["Hq"] * case["D"], case["Hkv"] * case["D"]
    bytes_ = 2 * q * size + 2 * _rows_read(case) * kv * size + sum(new) * case["Hq"] * 4
    flops = 4 * case["D"] * case["Hq"] * _pairs(case)
    if case["kind"] == "step":          # and dO, dQ; dK, dV in the model's type
        bytes_ += 2 * q * size + 2 * _rows_read(case) * kv * size
        flops = flops * 14 // 4
    if case["kind"] == "serve" and case["append"]:
        bytes_ += 4 * sum(new) * kv * size
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    new, kept = _lengths(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, Hq, Hkv, D = TYPES[case["dtype"]], case["Hq"], case["Hkv"], case["D"]
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dt)
    ints = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)
    T = sum(new)
    ends = [a + b for a, b in zip(new, kept)]
    s = dict(case=case, new=new, kept=kept, scale=1.0 / math.sqrt(D))
    if case["kind"] == "serve":
        qkv = rnd(T, Hq + 2 * Hkv, D)
        page = case["page"]
        width = max(-(-n // page) for n in ends)
        table = np.full((len(new), width), -1, dtype=np.int32)
        held = []
        for i, (a, b) in enumerate(zip(new, kept)):
            first = max(0, b + 1 - case["window"]) // page if case["window"] else 0
            held += [(i, p) for p in range(-(-ends[i] // page)) if p >= first or p * page < case["sinks"]]
        order = np.random.default_rng([seed, 5]).permutation(len(held) + 3)[:len(held)]
        for (i, p), at in zip(held, order):
            table[i, p] = at
        s.update(k_pages=rnd(len(held) + 3, page, Hkv, D), v_pages=rnd(len(held) + 3, page, Hkv, D), block_table=ints(table),
                 kv_lens=ints(ends), longest=max(ends))
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    elif case["packed"]:
        qkv = rnd(T, Hq + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    else:
        s["q"], s["k"], s["v"] = rnd(T, Hq, D), rnd(sum(ends), Hkv, D), rnd(sum(ends), Hkv, D)
    s["cu_q"], s["cu_k"] = ints(np.cumsum([0] + new)), ints(np.cumsum([0] + ends))
    s["o"], s["lse"] = torch.empty(T, Hq, D, device=DEV, dtype=dt), torch.empty(Hq, T, device=DEV)
    if case["kind"] == "step":
        s["d_o"], s["d_q"] = rnd(T, Hq, D), torch.empty(T, Hq, D, device=DEV, dtype=dt)
        s["d_kv"] = torch.empty(2, sum(ends), Hkv, D, device=DEV)
    s["blocks"] = _blocks(case, new, ends)
    return s


def _blocks(case, new, ends):
    """Which rows and keys the plain form takes together: blocks of rows of one sequence, and for each block the positions of the sinks and
    of the longest stretch of keys that one of its rows can see."""
    n = _block_rows(case)
    first_row, starts = np.cumsum([0] + new), np.cumsum([0] + ends)
    rows, pos, seq, low = [], [], [], []
    for i, (a, e) in enumerate(zip(new, ends)):
        for r in range(0, a, n):
            at = np.arange(r, r + n)
            rows.append(np.where(at < a, first_row[i] + at, -1))
            pos.append(e - a + at)
            seq.append(i)
            low.append(max(0, e - a + r - case["window"] + 1) if case["window"] else 0)
    far = max(ends)
    wide = min(far, case["window"] + n - 1) if case["window"] else far
    sinks = min(case["sinks"], far) if case["window"] else 0
    low, end = np.array(low)[:, None], np.array(ends)[seq][:, None]
    keys = np.concatenate([np.where(np.arange(sinks)[None] < low, np.arange(sinks)[None], far), low + np.arange(wide)[None]], axis=1)
    keys = np.where(keys < end, keys, -1)              # -1: no key
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return dict(rows=to(np.stack(rows)), pos=to(np.stack(pos)), seq=to(np.array(seq)), keys=to(keys.astype(np.int64)),
                start=to(starts[seq][:, None].astype(np.int64)))


# ---------------------------------------------------------------------------------------------------- plain forms
def _visible(s):
    b, c = s["blocks"], s["case"]
    p, j = b["pos"][:, :, None], b["keys"][:, None, :]
    seen = (j >= 0) & (j <= p) & (b["rows"] >= 0)[:, :, None]
    return seen & ((j > p - c["window"]) | (j < c["sinks"])) if c["window"] else seen


def _plain_append(s):
    b, page = s["blocks"], s["case"]["page"]
    at, ok = b["pos"], b["rows"] >= 0
    where = s["block_table"].long()[b["seq"][:, None].expand_as(at)[ok], at[ok] // page] * page + at[ok] % page
    for pages, x in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        pages.view(-1, *pages.shape[2:])[where] = x[b["rows"][ok]]


def _plain(s, backward):
    c, b = s["case"], s["blocks"]
    G, D = c["Hq"] // c["Hkv"], c["D"]
    seen, ok, rows = _visible(s), b["rows"] >= 0, b["rows"].clamp(min=0)
    if c["kind"] == "serve":
        page = c["page"]
        number = s["block_table"].long()[b["seq"]].gather(1, b["keys"].clamp(min=0) // page)
        seen = seen & (number >= 0)[:, None, :]
        at = number.clamp(min=0) * page + b["keys"].clamp(min=0) % page
        keys, values = s["k_pages"].view(-1, c["Hkv"], D), s["v_pages"].view(-1, c["Hkv"], D)
    else:
        at, keys, values = b["start"] + b["keys"].clamp(min=0), s["k"], s["v"]
    n, m = rows.shape
    seen = seen[:, None]                                # [blocks, heads of a group, rows, keys]
    if backward:
        d_k, d_v = s["d_kv"].zero_()
    group = lambda x, h: x[rows, h * G:(h + 1) * G].float().permute(0, 2, 1, 3).reshape(n, G * m, D)
    back = lambda x: x.reshape(n, G, m, D).permute(0, 2, 1, 3)[ok]
    for h in range(c["Hkv"]):
        q, k, v = group(s["q"], h), keys[at, h].float(), values[at, h].float()
        x = (torch.matmul(q, k.transpose(1, 2)) * s["scale"]).view(n, G, m, -1).masked_fill(~seen, -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        x = torch.exp(x - top)
        total = x.sum(-1, keepdim=True)
        p = (x / torch.where(total == 0, 1.0, total)).view(n, G * m, -1)
        heads = slice(h * G, (h + 1) * G)
        s["o"][b["rows"][ok], heads] = back(torch.matmul(p, v)).to(s["o"].dtype)
        s["lse"][heads, b["rows"][ok]] = (top + torch.log(total))[..., 0].permute(0, 2, 1)[ok].t()
        if backward:
            d_o = group(s["d_o"], h)
            d_v[:, h].index_add_(0, at.reshape(-1), torch.matmul(p.transpose(1, 2), d_o).reshape(-1, D))
            d_p = torch.matmul(d_o, v.transpose(1, 2))
            d_s = p * (d_p - (p * d_p).sum(-1, keepdim=True))
            s["d_q"][b["rows"][ok], heads] = back(torch.matmul(d_s, k) * s["scale"]).to(s["d_q"].dtype)
            d_k[:, h].index_add_(0, at.reshape(-1), torch.matmul(d_s.transpose(1, 2), q).reshape(-1, D) * s["scale"])


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _call(s):
    """The arguments of the calls, as a program lays them out once for its buffers."""
    from paper_2503_02356_amd import binding as B
    c = s["case"]
    call = {"B": B}
    if c["kind"] == "serve":
        call["append"] = B.make_kv_append_params(s["k"], s["v"], s["k_pages"], s["v_pages"], s["cu_q"], s["kv_lens"], s["block_table"])
        call["paged"] = B.make_paged_params(s["q"], s["k_pages"], s["v_pages"], s["o"], s["lse"], s["cu_q"], s["kv_lens"], s["block_table"],
                                            s["scale"], max_kv_len=s["longest"], window=c["window"], n_sinks=c["sinks"])
    else:
        call["fwd"] = B.make_fwd_params(s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu_q"], s["cu_k"], s["scale"])
        if c["kind"] == "step":
            ws = torch.empty(B.cf_attn_window_bwd_workspace_bytes(call["fwd"], c["window"], c["sinks"]), dtype=torch.uint8, device=DEV)
            call["bwd"] = B.make_bwd_params(call["fwd"], s["d_o"], s["d_q"], s["d_kv"][0], s["d_kv"][1], ws)
    return call


def run(state):
    s, c = state, state["case"]
    if own:
        if "call" not in s:
            s["call"] = _call(s)
        call = s["call"]
        B = call["B"]
        if c["kind"] == "serve":
            if c["append"]:
                B.cf_kv_append(call["append"])
            B.cf_attn_paged_fwd(call["paged"])
        else:
            B.cf_attn_window_fwd(call["fwd"], c["window"], c["sinks"])
            if c["kind"] == "step":
                s["d_kv"].zero_()
                B.cf_attn_window_bwd(call["bwd"], c["window"], c["sinks"])
    else:
        if c["kind"] == "serve" and c["append"]:
            _plain_append(s)
        _plain(s, c["kind"] == "step")
    out = {"o": s["o"], "lse": s["lse"]}
    if c["kind"] == "step":
        d_k, d_v = s["d_kv"].to(s["q"].dtype)
        out.update(d_q=s["d_q"], d_k=d_k, d_v=d_v)
    if c["kind"] == "serve" and c["append"]:
        out.update(k_pages=s["k_pages"], v_pages=s["v_pages"])
    return out


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    """Sequence by sequence and head by head from the definition, gradients by differentiation."""
    new, kept = _lengths(case)
    if _pairs(case) * case["Hq"] > 3e10 or len(new) * case["Hq"] > 6000:
        return None
    s = prepare(case, seed)
    G, grad = case["Hq"] // case["Hkv"], case["kind"] == "step"
    o, lse = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    out = {"o": o, "lse": lse}
    if grad:
        out.update(d_q=torch.zeros_like(o), d_k=torch.zeros(s["k"].shape, dtype=torch.float64, device=DEV),
                   d_v=torch.zeros(s["k"].shape, dtype=torch.float64, device=DEV))
    if case["kind"] == "serve" and case["append"]:
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
    row = key = 0
    for i, (a, b) in enumerate(zip(new, kept)):
        n, page = a + b, case.get("page")
        if page is None:
            keys, values, held = s["k"][key:key + n], s["v"][key:key + n], torch.ones(n, dtype=torch.bool, device=DEV)
        else:
            slots = s["block_table"][i, :-(-n // page)].long()
            held = (slots >= 0).repeat_interleave(page)[:n]
            where = ((slots.clamp(min=0) * page)[:, None] + torch.arange(page, device=DEV)).reshape(-1)[:n]
            keys, values = s["k_pages"].flatten(0, 1)[where], s["v_pages"].flatten(0, 1)[where]
            if case["append"]:
                keys[b:], values[b:] = s["k"][row:row + a], s["v"][row:row + a]
                kp.flatten(0, 1)[where[b:]], vp.flatten(0, 1)[where[b:]] = s["k"][row:row + a].double(), s["v"][row:row + a].double()
        for h in range(case["Hq"]):
            kh = h // G
            for r in range(0, a, 2048):
                e = min(a, r + 2048)
                lo = max(0, b + r + 1 - case["window"]) if case["window"] else 0
                j = torch.cat([torch.arange(min(lo, case["sinks"]), device=DEV), torch.arange(lo, b + e, device=DEV)])
                p = torch.arange(b + r, b + e, device=DEV)[:, None]
                hidden = (j[None] > p) | ~held[j][None]
                if case["window"]:
                    hidden |= (p - j[None] >= case["window"]) & (j[None] >= case["sinks"])
                with torch.set_grad_enabled(grad):
                    q, k, v = (x.double().requires_grad_(grad) for x in (s["q"][row + r:row + e, h], keys[j, kh], values[j, kh]))
                    score = ((q @ k.T) * s["scale"]).masked_fill(hidden, -math.inf)
                    y = torch.softmax(score, dim=-1) @ v
                    lse[h, row + r:row + e] = torch.logsumexp(score, dim=-1).detach()
                    o[row + r:row + e, h] = y.detach()
                    if grad:
                        d = torch.autograd.grad(y, (q, k, v), s["d_o"][row + r:row + e, h].double())
                        out["d_q"][row + r:row + e, h] = d[0]
                        out["d_k"][key + j, kh] += d[1]
                        out["d_v"][key + j, kh] += d[2]
        row, key = row + a, key + n
    if case["kind"] == "serve" and case["append"]:
        out.update(k_pages=kp, v_pages=vp)
    return out
