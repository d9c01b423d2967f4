"""Key/value pages of many sequences, and the forward passes of a chunk plan over them (evaluating or serving what has been trained).

Memory placement and descriptors only -- every arithmetic step runs inside cf_attn_paged_fwd and cf_attn_paged8_fwd, every copy inside cf_kv_append,
cf_kv_append_rotated and cf_kv_append8.
The runner's state buffers hold a split sequence's keys and values in one contiguous piece of its full length, for as long as gradients
are to be added to it.  Forward passes alone need no such piece: here a sequence takes pages from a pool as it grows, in any order, gives them
back when it is done, and with a window those that no later query sees, so that a window bounds the pages that a sequence of any length holds.  (Its
row of the table, 4 bytes a page, stays as long as the sequence, and goes to the GPU with every call.)
"""
import numpy as np
import torch

from . import binding as B


class PagedCache:
    """A pool of n_pages pages of page_size tokens and the tables of the sequences that live in it.

    window, n_sinks: of every call (0: a query sees all keys before it); pages behind the window of a sequence's next token are given back
    as soon as the tokens up to it have attended.
    eight_bits: keys and values are held in 8 bits, with a power of two for each 16 tokens of a page and head (k_scales, v_scales); dtype is that of the
    tensors that attend() takes.
    rotation (binding.make_rotation): attend() rotates keys and queries by their positions; without it they come rotated, where they are to be.
    A call lays its tables out on the host and copies them: a program that captures its steps into a graph keeps tables of its own and makes the two
    calls of the binding (cf_kv_append, cf_attn_paged_fwd, or those of their kind) itself."""

    def __init__(self, n_pages, page_size, n_kv_heads, head_dim, dtype=torch.bfloat16, device="cuda:0", window=0, n_sinks=0, eight_bits=False, rotation=None):
        self.page_size, self.window, self.n_sinks, self.dev = int(page_size), int(window), int(n_sinks), torch.device(device)
        self.dtype, self.eight_bits, self.rotation = dtype, bool(eight_bits), rotation
        self.k_pages = torch.empty((n_pages, page_size, n_kv_heads, head_dim), dtype=torch.float8_e4m3fn if eight_bits else dtype, device=self.dev)
        self.v_pages = torch.empty_like(self.k_pages)
        if eight_bits:
            if page_size % B.CF_KV8_BLOCK:
                raise ValueError(f"pages of {page_size} tokens do not hold whole blocks of {B.CF_KV8_BLOCK}")
            self.k_scales = torch.empty((n_pages, n_kv_heads, page_size // B.CF_KV8_BLOCK), dtype=torch.float32, device=self.dev)
            self.v_scales = torch.empty_like(self.k_scales)
        self.free = list(range(n_pages - 1, -1, -1))
        self.seqs = {}                               # name -> [length, pages (-1: given back)]
        self.peak_pages = 0

    def used_pages(self):
        return self.k_pages.shape[0] - len(self.free)

    def lengths(self):
        return {name: s[0] for name, s in self.seqs.items()}

    def close(self, name):
        """Gives a sequence's pages back."""
        self.free += [p for p in self.seqs.pop(name)[1] if p >= 0]

    def _grow(self, names, counts):
        """Room for counts[i] more tokens of names[i]; nothing changes where there is not enough."""
        need = {}
        for name, n in zip(names, counts):
            if n < 0 or name in need:
                raise ValueError("a batch names a sequence once and adds no negative number of tokens")
            length, pages = self.seqs.get(name, (0, []))
            need[name] = -(-(length + n) // self.page_size) - len(pages)
        if sum(need.values()) > len(self.free):
            raise MemoryError(f"{sum(need.values())} pages needed, {len(self.free)} free")
        for name, n in zip(names, counts):
            s = self.seqs.setdefault(name, [0, []])
            s[0] += int(n)
            s[1] += [self.free.pop() for _ in range(need[name])]
        self.peak_pages = max(self.peak_pages, self.used_pages())

    def _give_back(self, names):
        kept = -(-self.n_sinks // self.page_size)    # columns with sinks
        for name in names:
            length, pages = self.seqs[name]
            first = length - self.window + 1         # the first key that the next token's window holds
            begin = end = min(len(pages), max(0, first) // self.page_size)
            while begin > kept and pages[begin - 1] >= 0:        # (those before it have been given back)
                begin -= 1
            for c in range(begin, end):
                self.free.append(pages[c])
                pages[c] = -1

    def attend(self, names, counts, q, k, v, scale=None, lse=None):
        """counts[i] new tokens of sequence names[i] (new names begin a sequence), their rows one behind the other in q [T,Hq,D] and k, v
        [T,Hkv,D]: their keys and values are written into pages, then they attend to all that their sequences hold.  -> o [T,Hq,D] (rows
        behind the last sequence's, of a padded batch, 0), in the order of the current stream; lse: [Hq,T] fp32 tensor to be written, or
        None.  Raises MemoryError where pages are missing; whatever it raises, the sequences are what they were."""
        names, counts = list(names), [int(n) for n in counts]
        if not names or len(names) != len(counts):
            raise ValueError(f"{len(names)} sequences and {len(counts)} numbers of new tokens")
        if sum(counts) > q.shape[0] or q.shape[0] != k.shape[0]:
            raise ValueError(f"{sum(counts)} new tokens in {q.shape[0]} rows of q and {k.shape[0]} of k")
        before = {name: (self.seqs[name][0], len(self.seqs[name][1])) for name in names if name in self.seqs}
        self._grow(names, counts)
        try:
            o = self._append_and_attend(names, counts, q, k, v, scale, lse)
        except Exception:
            for name in reversed(names):             # (arguments that the calls refuse)
                length, n = before.get(name, (0, 0))
                pages = self.seqs[name][1]
                self.free += reversed(pages[n:])
                self.seqs[name] = [length, pages[:n]]
                if name not in before:
                    del self.seqs[name]
            raise
        if self.window:
            self._give_back(names)
        return o

    def _append_and_attend(self, names, counts, q, k, v, scale, lse):
        held = [self.seqs[name] for name in names]
        table = np.full((len(names), max(1, max(len(pages) for _, pages in held))), -1, dtype=np.int32)
        for i, (_, pages) in enumerate(held):
            table[i, :len(pages)] = pages
        lens = np.array([length for length, _ in held], dtype=np.int32)
        # one copy: bounds, lengths, table
        desc = torch.from_numpy(np.concatenate([np.cumsum([0] + counts).astype(np.int32), lens, table.reshape(-1)])).to(self.dev)
        n = len(names)
        cu, kv_lens, block_table = desc[:n + 1], desc[n + 1:2 * n + 1], desc[2 * n + 1:].view(table.shape)
        o = torch.empty_like(q) if sum(counts) == q.shape[0] else torch.zeros_like(q)
        where, scale = (cu, kv_lens, block_table), scale if scale is not None else q.shape[2] ** -0.5
        how = dict(max_kv_len=int(lens.max()), window=self.window, n_sinks=self.n_sinks)
        turn, queries = None, q
        if self.rotation is not None:
            queries = torch.empty_like(q)            # (the caller's stay)
            turn = B.make_append_rotation(self.rotation, q, queries)
        if self.eight_bits:
            assert q.dtype == self.dtype
            cache = (self.k_pages, self.v_pages, self.k_scales, self.v_scales)
            append = B.make_kv_append8_params(k, v, *cache, *where)
            attention = B.make_paged8_params(queries, *cache, o, lse, *where, scale, **how)
            if B.paged8_refuses(attention):
                # (the append may round older rows again: what the attention would refuse is refused before)
                raise ValueError("q and lse must be aligned, with strides of at least head_dim that are, and scale a finite fp32 number")
            B.cf_kv_append8(append, turn)
            B.cf_attn_paged8_fwd(attention)
            return o
        append = B.make_kv_append_params(k, v, self.k_pages, self.v_pages, *where)
        attention = B.make_paged_params(queries, self.k_pages, self.v_pages, o, lse, *where, scale, **how)
        if turn is None:
            B.cf_kv_append(append)
        else:
            B.cf_kv_append_rotated(append, turn)
        B.cf_attn_paged_fwd(attention)
        return o


def plan_forward(plan, cache, inputs, scale=None):
    """Forward passes of a plan's chunks over a cache, in the order of section 4.2 (a group's chunks ascending); a group's sequences leave
    the cache behind its last chunk, or where the passes end before it.  inputs(chunk) -> q [T,Hq,D], k, v [T,Hkv,D] of the chunk's tokens on the
    device.  Yields (chunk, o, lse).  The cache may hold other sequences, under any names: they stay as they are (the plan's have names that
    nobody else has)."""
    run = object()
    for g in range(plan.n_groups):
        names = {}                                   # of the group, in the order of their beginnings
        try:
            for c in plan.group(g):
                segs = plan.chunk_segments(int(c))
                q, k, v = inputs(int(c))
                lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
                own = [(run, sid) for sid, _, _ in segs]
                names.update(dict.fromkeys(own))
                yield int(c), cache.attend(own, [n for _, _, n in segs], q, k, v, scale, lse), lse
        finally:
            for name in names:
                if name in cache.seqs:
                    cache.close(name)
