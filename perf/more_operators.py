"""The work of the position rotation and of the calls on an 8-bit key/value cache, as a training and as a serving program makes them.

Kinds of a case
  rotate   queries and keys of one training chunk are rotated by their positions, and the gradients of the rotated ones are rotated back: dQ in
           the model's type, dK, which the attention accumulates in 32 bits, to the model's type.
  append   new tokens' keys, rotated, and their values go into the pages of a cache of the model's type; their queries are rotated.
  append8  the same into a cache of 8 bits.
  attend8  new tokens' queries attend over a cache of 8 bits.
  serve8   append8, then attend8, as one layer of a serving step makes them.

Rotation: elements (i, i + rot/2) of a head, or (2i, 2i+1) where interleaved, turn by position * inv_freq[i]; those from `rot` on stay.
Cache of 8 bits: values of the e4m3 format in pages [pages][tokens][heads][D] and for each 16 tokens of a page and each head a power of two that
they are multiplied with: the least that keeps all of the block's values within 448.  A block that new tokens are added to keeps its power or
takes a larger one, to which its older values are rounded again.
A query at position p of its sequence sees the keys j <= p with j > p - window (window 0: all) or j < sinks.
Sequence lengths are drawn from the case alone (lens_seed), values from the seed that prepare() is given.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
E4M3 = torch.float8_e4m3fn
BLOCK = 16                   # tokens that share a power of two
LEAST = -110                 # exponent of the smallest one


def _chunk(name, dtype, Hq, Hkv, D, T, prefix, median, rot, interleaved=False, lens_seed=0):
    """median > 0: T tokens of packed sequences, lognormal (sigma 0.9) around it; 0: one slice of T tokens behind `prefix` others."""
    c = dict(kind="rotate", dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, T=T, prefix=prefix, median=median, rot=rot, interleaved=interleaved, lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def _serve(name, kind, dtype, Hq, Hkv, D, page, n_tokens, n_chunks, chunk, least, most, rot, interleaved=False, window=0, sinks=0, lens_seed=0):
    """n_tokens sequences with one new token, n_chunks with `chunk` new tokens (each, a little fewer in every other one), behind `least` to
    `most` cached tokens, in pages of `page` tokens."""
    c = dict(kind=kind, dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, page=page, n_tokens=n_tokens, n_chunks=n_chunks, chunk=chunk, least=least, most=most,
             rot=rot, interleaved=interleaved, window=window, sinks=sinks, lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a layer checked in full precision: one short slice
        _chunk("rotate_fp32_slice", "fp32", 6, 2, 128, 333, 1000, 0, 128),
        # a packed chunk of the 8K configuration
        _chunk("rotate_packed_8k", "bf16", 28, 4, 128, 8192, 0, 600, 128),
        # the last slice of the 256K configuration, pairs next to each other, a part of the head rotated
        _chunk("rotate_256k_slice", "bf16", 64, 8, 128, 32768, 229376, 0, 64, True),
        # one conversation, one token, into a cache of the model's type
        _serve("append_token_1", "append", "bf16", 28, 4, 128, 16, 1, 0, 0, 4097, 4097, 128),
        # a chunk of a long prompt into such a cache
        _serve("append_prompt_8k", "append", "bf16", 28, 4, 128, 64, 0, 1, 8192, 24579, 24579, 128),
        # the same chunk into 8 bits
        _serve("append8_prompt_8k", "append8", "bf16", 28, 4, 128, 64, 0, 1, 8192, 24579, 24579, 128),
        # one token of each conversation of a large batch, blocks filled to any degree
        _serve("append8_tokens_256", "append8", "bf16", 16, 4, 64, 32, 256, 0, 0, 100, 20000, 64, True),
        # one layer of a step of one conversation
        _serve("serve8_token_1", "serve8", "bf16", 28, 4, 128, 16, 1, 0, 0, 4097, 4097, 128),
        # a batch of conversations of different lengths
        _serve("attend8_tokens_64", "attend8", "bf16", 32, 8, 128, 64, 64, 0, 0, 500, 16384, 128),
        # a large batch of a model with windowed layers: pages behind the window have been given back
        _serve("serve8_tokens_256_window", "serve8", "bf16", 16, 4, 64, 32, 256, 0, 0, 100, 20000, 64, window=1024, sinks=4),
        # a chunk of a long prompt
        _serve("attend8_prompt_32k", "attend8", "bf16", 28, 4, 128, 64, 0, 1, 8192, 24576, 24576, 128),
        # tokens and chunks of prompts in one step, checked in full precision
        _serve("serve8_fp32_mixed", "serve8", "fp32", 6, 2, 128, 16, 3, 2, 100, 20, 700, 96),
    ]


_HEADS = [(28, 4), (32, 8), (64, 8), (16, 2), (8, 2), (4, 4), (14, 2), (16, 16)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: at most the arithmetic of attend8_prompt_32k, the bytes of rotate_256k_slice, a cache of 1 GB."""
    seed = rng.randrange(1, 1 << 30)
    kind = rng.choice(["rotate", "rotate", "append", "append", "append8", "append8", "attend8", "attend8", "attend8", "serve8", "serve8", "serve8"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        D = rng.choice([64, 128, 128])
        rot = rng.choice([D, D, D // 2, 16 * rng.randint(1, D // 16)])
        Hq, Hkv = rng.choice(_HEADS) if dtype == "bf16" else rng.choice([(1, 1), (4, 4), (6, 2), (8, 2)])
        if kind == "rotate":
            T = _log(rng, 1, 32768 if dtype == "bf16" else 4000)
            median = rng.choice([0, 0, _log(rng, 20, 2000)])
            prefix = 0 if median else rng.choice([0, _log(rng, 1, 229376)])
            c = _chunk("", dtype, Hq, Hkv, D, T, prefix, median, rot, rng.random() < 0.4, seed)
        else:
            shape = rng.choice(["tokens", "tokens", "prompt", "mixed"])
            one = 0 if shape == "prompt" else _log(rng, 1, 256)
            chunks = 0 if shape == "tokens" else rng.randint(1, 3)
            most = _log(rng, 1, 60000 if dtype == "bf16" else 5000)
            window = rng.choice([0, 0, _log(rng, 1, 8192)])
            sinks = rng.choice([0, 1, 4, 4, 16, 64, 200]) if window else 0
            c = _serve("", kind, dtype, Hq, Hkv, D, rng.choice([16, 32, 64, 128, 256]), one, chunks, _log(rng, 2, 4096 if dtype == "bf16" else 300),
                       max(0, int(most * rng.random())), most, rot, rng.random() < 0.4, window, sinks, seed)
            new, kept = _lengths(c)
            if (sum(new) + sum(kept)) * Hkv * D * 2 * (1 if kind != "append" else 4 if dtype == "fp32" else 2) > 1 << 30:
                continue
        w = work(c)
        if w["flops"] > (2e12 if dtype == "bf16" else 2e11) or w["bytes"] > 2.4e9:
            continue
        if kind in ("attend8", "serve8"):
            widest = max(a + b for a, b in zip(new, kept))
            widest = min(widest, c["window"] + 400) if c["window"] else widest
            rows = sum(-(-n // _block_rows(c)) for n in new) * _block_rows(c)
            if rows * (Hq // Hkv) * widest * 4 > 6 << 30:
                continue
        return c


def _lengths(case):
    """(new tokens, tokens before them) of each sequence."""
    rng = random.Random(case["lens_seed"] * 7919 + 13)
    if case["kind"] != "rotate":
        new = [1] * case["n_tokens"] + [max(1, case["chunk"] - (37 * (i % 2) if case["chunk"] > 64 else 0)) for i in range(case["n_chunks"])]
        return new, [rng.randint(case["least"], max(case["least"], case["most"])) for _ in new]
    if case["median"] == 0:
        return [case["T"]], [case["prefix"]]
    new, left = [], case["T"]
    while left > 0:
        n = min(left, max(1, int(round(math.exp(rng.gauss(math.log(case["median"]), 0.9))))))
        new.append(n)
        left -= n
    return new, [0] * len(new)


def _block_rows(case):
    """Rows that the plain form of the attention takes together."""
    return 1 if case["n_chunks"] == 0 else 32 if case["n_tokens"] > 0 else 128


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
    kind, size = case["kind"], 2 if case["dtype"] == "bf16" else 4
    T = sum(_lengths(case)[0])
    q, kv = T * case["Hq"] * case["D"], T * case["Hkv"] * case["D"]
    bytes_ = flops = 0
    if kind == "rotate":                        # q, k there; dq and, from 32 bits, dk back
        bytes_ = 4 * q * size + 3 * kv * size + 4 * kv
        flops = 6 * (q + kv)
    if kind in ("append", "append8", "serve8"):
        held = 2 * kv * size if kind == "append" else 2 * kv + 2 * kv // case["D"] * 4 // BLOCK
        bytes_ += 2 * q * size + 2 * kv * size + held
        flops += 3 * (q + kv) + (0 if kind == "append" else 4 * kv)
    if kind in ("attend8", "serve8"):
        row = case["Hkv"] * case["D"]
        bytes_ += 2 * q * size + T * case["Hq"] * 4 + 2 * _rows_read(case) * (row + case["Hkv"] * 4 / BLOCK)
        flops += 4 * case["D"] * case["Hq"] * _pairs(case)
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    new, kept = _lengths(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, kind, Hq, Hkv, D = TYPES[case["dtype"]], case["kind"], case["Hq"], case["Hkv"], case["D"]
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dt)
    ints = lambda a: torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)
    T = sum(new)
    ends = [a + b for a, b in zip(new, kept)]
    s = dict(case=case, new=new, kept=kept, scale=1.0 / math.sqrt(D))
    half = case["rot"] // 2
    s["inv_freq"] = (10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
    s["position"] = torch.from_numpy(np.concatenate([np.arange(b, a + b) for a, b in zip(new, kept)])).to(DEV)
    s["cu_q"] = ints(np.cumsum([0] + new))
    qkv = rnd(T, Hq + 2 * Hkv, D)               # as one projection leaves them
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["q_out"] = torch.empty(T, Hq, D, device=DEV, dtype=dt)
    if kind == "rotate":
        s["cu_k"] = ints(np.cumsum([0] + ends))
        s["k_out"] = torch.empty(T, Hkv, D, device=DEV, dtype=dt)
        s["d_q"], s["d_q_out"] = rnd(T, Hq, D), torch.empty(T, Hq, D, device=DEV, dtype=dt)
        s["d_k"], s["d_k_out"] = torch.randn(T, Hkv, D, generator=g, device=DEV), torch.empty(T, Hkv, D, device=DEV, dtype=dt)
        return s
    page = case["page"]
    table = np.full((len(new), max(-(-n // page) for n in ends)), -1, dtype=np.int32)
    held = []
    for i, (a, b) in enumerate(zip(new, kept)):
        first = max(0, b + 1 - case["window"]) // page if case["window"] else 0
        held += [(i, p) for p in range(-(-ends[i] // page)) if p >= first or p * page < case["sinks"]]
    order = np.random.default_rng([seed, 5]).permutation(len(held) + 3)[:len(held)]
    for (i, p), at in zip(held, order):
        table[i, p] = at
    s.update(block_table=ints(table), kv_lens=ints(ends), longest=max(ends))
    n = len(held) + 3
    if kind == "append":
        s.update(k_pages=rnd(n, page, Hkv, D), v_pages=rnd(n, page, Hkv, D), sequence=_to(np.repeat(np.arange(len(new)), new)))
    else:
        for x in ("k", "v"):                    # blocks of different sizes, as the layers of a model give them
            values = torch.randn(n, page // BLOCK, BLOCK, Hkv, D, generator=g, device=DEV)
            values *= torch.exp(0.5 * torch.randn(n, page // BLOCK, 1, Hkv, 1, generator=g, device=DEV))
            power = _power(values.abs().amax((2, 4)))
            s[x + "_pages"] = (values / power[:, :, None, :, None]).to(E4M3).view(n, page, Hkv, D)
            s[x + "_scales"] = power.transpose(1, 2).contiguous()          # [pages][heads][blocks of a page]
            del values
        s["touched"] = _touched(new, ends, table, page)
    s["o"], s["lse"] = torch.empty(T, Hq, D, device=DEV, dtype=dt), torch.empty(Hq, T, device=DEV)
    s["blocks"] = _blocks(case, new, ends)
    return s


def _to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _touched(new, ends, table, page):
    """The blocks of 16 tokens that get new ones: their page and block of it, for each of their 16 places the new row (-1: none), and whether
    older rows stand before the new ones."""
    pages, blocks, rows, older = [], [], [], []
    first_row = 0
    for i, (a, e) in enumerate(zip(new, ends)):
        for b in range((e - a) // BLOCK, -(-e // BLOCK)):
            pages.append(table[i, b * BLOCK // page])
            blocks.append(b % (page // BLOCK))
            at = b * BLOCK + np.arange(BLOCK) - (e - a)
            rows.append(np.where((at >= 0) & (at < a), first_row + at, -1))
            older.append(at < 0)
        first_row += a
    return dict(page=_to(np.array(pages, dtype=np.int64)), block=_to(np.array(blocks, dtype=np.int64)), rows=_to(np.stack(rows)), older=_to(np.stack(older)))


def _blocks(case, new, ends):
    """Which rows and keys the plain form of the attention takes together: blocks of rows of one sequence, and for each block the positions of
    the sinks and of the longest stretch of keys that one of its rows can see."""
    if case["kind"] not in ("attend8", "serve8"):
        return None
    n = _block_rows(case)
    first_row = np.cumsum([0] + new)
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
    return dict(rows=_to(np.stack(rows)), pos=_to(np.stack(pos)), seq=_to(np.array(seq)), keys=_to(keys.astype(np.int64)))


# ---------------------------------------------------------------------------------------------------- plain forms
def _turned(s, x, back=False):
    """x [T,H,D] in 32 bits, turned by the rows' positions."""
    rot, half = s["case"]["rot"], s["case"]["rot"] // 2
    x = x.float()
    angle = s["position"].double()[:, None] * s["inv_freq"].double()[None]
    c, d = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None] * (-1 if back else 1)
    y = x.clone()
    if s["case"]["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * d, a * d + b * c
    else:
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half], y[..., half:rot] = a * c - b * d, a * d + b * c
    return y


def _power(most):
    """The least power of two, from 2^LEAST on, 448 times which is not less than `most`."""
    m, e = torch.frexp(most)                       # most = m 2^e, m from 0.5 on
    e = torch.where(most == 0, LEAST, e - 9 + (m > 0.875).int()).clamp(min=LEAST)
    return ((e + 127) << 23).view(torch.float32)   # (from its bits: a power function need not be exact)


def _plain_append(s):
    where = s["block_table"].long()[s["sequence"], s["position"] // s["case"]["page"]]
    at = where * s["case"]["page"] + s["position"] % s["case"]["page"]
    for pages, x in ((s["k_pages"], _turned(s, s["k"])), (s["v_pages"], s["v"])):
        pages.view(-1, *pages.shape[2:])[at] = x.to(pages.dtype)


def _plain_append8(s):
    t = s["touched"]
    page, rows = t["page"], t["rows"]
    fresh, older = (rows >= 0)[:, :, None, None], t["older"][:, :, None, None]
    for x, name in ((_turned(s, s["k"]), "k"), (s["v"].float(), "v")):
        codes = s[name + "_pages"].view(torch.uint8).view(-1, s["case"]["page"] // BLOCK, BLOCK, *x.shape[1:])
        scales = s[name + "_scales"].transpose(1, 2)
        had, old = codes[page, t["block"]], scales[page, t["block"]]                     # [blocks, 16, heads, D], [blocks, heads]
        values = torch.where(fresh, x[rows.clamp(min=0)], 0.0)
        power = _power(values.abs().amax((1, 3)))
        power = torch.where(t["older"][:, :1], torch.maximum(power, old), power)
        again = had.view(E4M3).float() * (old / power)[:, None, :, None]
        code = torch.where(fresh, values / power[:, None, :, None], again).to(E4M3).view(torch.uint8)
        codes[page, t["block"]] = torch.where(fresh | older, code, had)
        scales[page, t["block"]] = power


def _plain_attend8(s, queries):
    c, b = s["case"], s["blocks"]
    G, D, page = c["Hq"] // c["Hkv"], c["D"], c["page"]
    ok, rows = b["rows"] >= 0, b["rows"].clamp(min=0)
    p, j = b["pos"][:, :, None], b["keys"][:, None, :]
    seen = (j >= 0) & (j <= p) & ok[:, :, None]
    if c["window"]:
        seen &= (j > p - c["window"]) | (j < c["sinks"])
    keys = b["keys"].clamp(min=0)
    number = s["block_table"].long()[b["seq"]].gather(1, keys // page)
    seen = (seen & (number >= 0)[:, None, :])[:, None]                   # [blocks, heads of a group, rows, keys]
    number = number.clamp(min=0)
    n, m = rows.shape
    group = lambda x, h: x[rows, h * G:(h + 1) * G].float().permute(0, 2, 1, 3).reshape(n, G * m, D)
    back = lambda x: x.reshape(n, G, m, D).permute(0, 2, 1, 3)[ok]
    held = lambda x, h: (s[x + "_pages"].view(torch.uint8)[number, keys % page, h].view(E4M3).float()
                         * s[x + "_scales"][number, h, keys % page // BLOCK][..., None])
    for h in range(c["Hkv"]):
        heads = slice(h * G, (h + 1) * G)
        x = (torch.matmul(group(queries, h), held("k", h).transpose(1, 2)) * s["scale"]).view(n, G, m, -1).masked_fill(~seen, -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        x = torch.exp(x - top)
        total = x.sum(-1, keepdim=True)
        x = (x / torch.where(total == 0, 1.0, total)).view(n, G * m, -1)
        s["o"][b["rows"][ok], heads] = back(torch.matmul(x, held("v", h))).to(s["o"].dtype)
        s["lse"][heads, b["rows"][ok]] = (top + torch.log(total))[..., 0].permute(0, 2, 1)[ok].t()


def _plain(s):
    kind, dt = s["case"]["kind"], s["q"].dtype
    if kind == "rotate":
        s["q_out"].copy_(_turned(s, s["q"])), s["k_out"].copy_(_turned(s, s["k"]))
        s["d_q_out"].copy_(_turned(s, s["d_q"], True)), s["d_k_out"].copy_(_turned(s, s["d_k"], True))
        return
    if kind != "attend8":
        s["q_out"].copy_(_turned(s, s["q"]))
    if kind == "append":
        _plain_append(s)
    elif kind != "attend8":
        _plain_append8(s)
    if kind in ("attend8", "serve8"):
        _plain_attend8(s, s["q"] if kind == "attend8" else s["q_out"])


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _calls(s):
    """The arguments of the calls, as a program lays them out once for its buffers."""
    from paper_2503_02356_amd import binding as B
    c, kind, call = s["case"], s["case"]["kind"], {"B": B}
    rotation = B.make_rotation(s["inv_freq"], c["interleaved"])
    if kind == "rotate":
        call["there"] = B.make_rotate_params(s["cu_q"], s["cu_k"], rotation, q=(s["q"], s["q_out"]), k=(s["k"], s["k_out"]))
        call["back"] = B.make_rotate_params(s["cu_q"], s["cu_k"], rotation, q=(s["d_q"], s["d_q_out"]), k=(s["d_k"], s["d_k_out"]), inverse=True)
        return call
    where = (s["cu_q"], s["kv_lens"], s["block_table"])
    call["turn"] = B.make_append_rotation(rotation, s["q"], s["q_out"])
    if kind == "append":
        call["append"] = B.make_kv_append_params(s["k"], s["v"], s["k_pages"], s["v_pages"], *where)
        return call
    cache = (s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
    call["append8"] = B.make_kv_append8_params(s["k"], s["v"], *cache, *where)
    if kind in ("attend8", "serve8"):
        q = s["q"] if kind == "attend8" else s["q_out"]
        call["attend8"] = B.make_paged8_params(q, *cache, s["o"], s["lse"], *where, s["scale"], max_kv_len=s["longest"], window=c["window"],
                                               n_sinks=c["sinks"])
    return call


def _own(s):
    if "call" not in s:
        s["call"] = _calls(s)
    call, kind = s["call"], s["case"]["kind"]
    B = call["B"]
    if kind == "rotate":
        B.cf_rotate(call["there"])
        B.cf_rotate(call["back"])
    if kind == "append":
        B.cf_kv_append_rotated(call["append"], call["turn"])
    if kind in ("append8", "serve8"):
        B.cf_kv_append8(call["append8"], call["turn"])
    if kind in ("attend8", "serve8"):
        B.cf_attn_paged8_fwd(call["attend8"])


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        _own(s)
    else:
        _plain(s)
    if kind == "rotate":
        return {x: s[x] for x in ("q_out", "k_out", "d_q_out", "d_k_out")}
    out = {} if kind == "attend8" else {x: s[x] for x in ("q_out", "k_pages", "v_pages")}
    if kind in ("append8", "serve8"):
        out.update(k_scales=s["k_scales"], v_scales=s["v_scales"])
    if kind in ("attend8", "serve8"):
        out.update(o=s["o"], lse=s["lse"])
    return out


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_turned(case, inv_freq, position, x, back=False):
    """As complex numbers times exp(i angle)."""
    rot = case["rot"]
    x = x.double()
    part = x[..., :rot]
    pairs = part.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else part.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    angle = position.double()[:, None, None] * inv_freq.double()
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), -angle if back else angle)
    z = torch.view_as_real(z)
    part = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([part, x[..., rot:]], dim=-1)


def exact(case, seed):
    """From the definition, in 64 bits: what the cache holds in 8 bits before it is rounded to them, attention sequence by sequence and head by
    head (over what the cache holds)."""
    kind, (new, kept) = case["kind"], _lengths(case)
    attends = kind in ("attend8", "serve8")
    if attends and (_pairs(case) * case["Hq"] > 3e10 or len(new) * case["Hq"] > 6000):
        return None
    s = prepare(case, seed)
    turned = lambda x, back=False: _exact_turned(case, s["inv_freq"], s["position"], x, back)
    if kind == "rotate":
        return dict(q_out=turned(s["q"]), k_out=turned(s["k"]), d_q_out=turned(s["d_q"], True), d_k_out=turned(s["d_k"], True))
    out, queries = {}, s["q"].double()
    if kind != "attend8":
        out["q_out"] = turned(s["q"])
        queries = out["q_out"].to(s["q"].dtype).double()
    page, D, Hkv = case["page"], case["D"], case["Hkv"]
    held = {}                                      # what each place of the pages stands for, rounded; its block's power of two
    for name, x in (("k", turned(s["k"]) if kind != "attend8" else None), ("v", s["v"].double())):
        pages = s[name + "_pages"]
        if kind == "append":
            values = pages.double().flatten(0, 1)
            row = 0
            for i, (a, b) in enumerate(zip(new, kept)):
                at = torch.arange(b, a + b, device=DEV)
                values[s["block_table"][i].long()[at // page] * page + at % page] = x[row:row + a]
                row += a
            out[name + "_pages"] = values.view(pages.shape)
            continue
        codes, scales = pages.double(), s[name + "_scales"].double()
        if kind != "attend8":
            stored = codes.clone()
            row = 0
            for i, (a, b) in enumerate(zip(new, kept)):
                first, n = b // BLOCK, -(-(a + b) // BLOCK) - b // BLOCK
                at = torch.arange(first, first + n, device=DEV) * BLOCK
                number, block = s["block_table"][i].long()[at // page], at % page // BLOCK
                values = torch.zeros(n * BLOCK, Hkv, D, dtype=torch.float64, device=DEV)
                lead = b - first * BLOCK
                values[lead:lead + a] = x[row:row + a]
                most = values.view(n, BLOCK, Hkv, D).abs().amax((1, 3))
                e = torch.ceil(torch.log2(most / 448)).clamp(min=LEAST)          # (log2 of 0: LEAST)
                power = ((e.long() + 1023) << 52).view(torch.float64)
                power = torch.where(448 * power / 2 >= most, power / 2, torch.where(448 * power < most, power * 2, power)).clamp(min=2.0 ** LEAST)
                if lead:
                    before = scales[number[0], :, block[0]]
                    power[0] = torch.maximum(power[0], before)
                    places = slice(int(block[0]) * BLOCK, int(block[0]) * BLOCK + lead)
                    values[:lead] = codes[number[0], places] * before[:, None]
                scales[number, :, block] = power
                values /= power.repeat_interleave(BLOCK, 0)[:, :, None]
                at = torch.arange(b - lead, a + b, device=DEV)
                number = s["block_table"][i].long()[at // page]
                codes[number, at % page] = values[:lead + a]
                stored[number, at % page] = values[:lead + a].to(E4M3).double()
                row += a
            out[name + "_pages"], out[name + "_scales"] = codes, scales
            codes = stored
        held[name] = codes.flatten(0, 1), scales.transpose(1, 2).repeat_interleave(BLOCK, 1).flatten(0, 1)
    if not attends:
        return out
    G = case["Hq"] // Hkv
    o, lse = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for i, (a, b) in enumerate(zip(new, kept)):
        for r in range(0, a, 2048):
            e = min(a, r + 2048)
            lo = max(0, b + r + 1 - case["window"]) if case["window"] else 0
            j = torch.cat([torch.arange(min(lo, case["sinks"]), device=DEV), torch.arange(lo, b + e, device=DEV)])
            number = s["block_table"][i].long()[j // page]
            at = number.clamp(min=0) * page + j % page
            position = torch.arange(b + r, b + e, device=DEV)[:, None]
            hidden = (j[None] > position) | (number < 0)[None]
            if case["window"]:
                hidden |= (position - j[None] >= case["window"]) & (j[None] >= case["sinks"])
            for h in range(Hkv):
                k, v = (held[x][0][at, h] * held[x][1][at, h][:, None] for x in ("k", "v"))
                for head in range(h * G, (h + 1) * G):
                    score = ((queries[row + r:row + e, head] @ k.T) * s["scale"]).masked_fill(hidden, -math.inf)
                    o[row + r:row + e, head] = torch.softmax(score, dim=-1) @ v
                    lse[head, row + r:row + e] = torch.logsumexp(score, dim=-1)
        row += a
    out.update(o=o, lse=lse)
    return out
