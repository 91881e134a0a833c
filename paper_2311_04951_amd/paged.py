"""Decoding over a key-value cache in pages that is held to a budget (Sections 2, 4.2: past keys and values are kept instead of
recomputed; Section 4.4: the memory they take is what the caches compete for).  Pages and control flow only - every number is produced
by the library's kernels.

A pass appends its rows to the pages of every sequence, attends what these hold and adds up the attention weights that every
position receives (ss_paged_forward); when a sequence has filled what it may, every head of every layer goes back to the budget by
those sums (ss_paged_evict), and the pages behind it are free for other sequences.
"""
from __future__ import annotations

import time

import torch

from . import (Model, PagedKV, SpecVerifyError, ss_greedy_accept, ss_paged_evict, ss_paged_forward, ss_softmax, ss_speculative_accept)


class PagedCache:
    """Pages for `batch` sequences of a model, taken from one pool as sequences grow and given back as they shrink.  `kv` is what the
    library's calls take, `lengths` the host's copy of the lengths."""

    def __init__(self, model: Model, batch: int, n_pages: int, page_size: int = 64, max_pages: int = 0, weights: bool = True):
        s, dev, i32 = model.shape, torch.device("cuda", torch.cuda.current_device()), torch.int32
        dtype = torch.bfloat16 if s.dtype == "bf16" else torch.float32
        k, v = (torch.empty((s.n_layers, n_pages, s.n_heads, page_size, s.head_dim), dtype=dtype, device=dev) for _ in range(2))
        meta = (s.n_layers, n_pages, s.n_heads, page_size)
        self.page_size, self.max_pages = page_size, max_pages or n_pages
        self.free, self.pages, self.lengths = list(range(n_pages - 1, -1, -1)), [[] for _ in range(batch)], [0] * batch
        self.kv = PagedKV(k, v, torch.full((batch, self.max_pages), -1, dtype=i32, device=dev), torch.zeros(batch, dtype=i32, device=dev),
                          next_pos=torch.zeros(batch, dtype=i32, device=dev), weight=torch.zeros(meta, device=dev) if weights else None,
                          position=torch.zeros(meta, dtype=i32, device=dev) if weights else None, status=torch.zeros(1, dtype=i32, device=dev))

    def one(self, b: int) -> PagedKV:
        """Sequence b alone."""
        kv = self.kv
        return PagedKV(kv.k, kv.v, kv.page_table[b:b + 1], kv.length[b:b + 1], next_pos=kv.next_pos[b:b + 1], weight=kv.weight,
                       position=kv.position, status=kv.status)

    def resize(self, b: int, n: int):
        """Sequence b holds n positions now (the device's length is the calls' to move): takes the pages it lacks, gives back the rest."""
        need, have = -(-n // self.page_size), self.pages[b]
        if need > self.max_pages or need - len(have) > len(self.free):
            raise MemoryError(f"sequence {b}: {need} pages of {self.page_size} positions; {len(have)} taken, {len(self.free)} free, {self.max_pages} at most")
        if need != len(have):
            self.free += have[need:][::-1]
            del have[need:]
            have += [self.free.pop() for _ in range(need - len(have))]
            self.kv.page_table[b].copy_(torch.tensor(have + [-1] * (self.max_pages - need), dtype=torch.int32))
        self.lengths[b] = n


def budgeted_generate(target: Model, prompts, n_new: int, temperature: float, budget: int, u=None, keep_first: int = 4, keep_recent: int = 0,
                      page_size: int = 64, stats=None):
    """`prompts` (lists of token ids, any lengths from one token, with n_new at most the model's max_pos + 1) are continued by n_new tokens each, all of them in one batch, with at
    most `budget` cached positions per head behind every eviction and a page more in front of it.  temperature 0: the most probable
    token; else one drawn with the uniforms u [batch][n_new].  keep_recent: positions that are always kept (0: half of what
    keep_first leaves of the budget).  Returns a list of token lists; `stats` (a dict, optional) receives evictions, pages (most in use) and loop_seconds."""
    dev = torch.device("cuda")
    B, V = len(prompts), target.shape.vocab
    if not all(len(p) for p in prompts):
        raise ValueError("a prompt needs at least one token")
    if budget < 1 or keep_first < 0 or keep_recent < 0:
        raise ValueError(f"budget {budget}, keep_first {keep_first}, keep_recent {keep_recent}")
    last = max(len(p) for p in prompts) + n_new - 1                   # positions that the longest sequence feeds
    if last > target.max_pos:
        raise ValueError(f"{last} positions of a model whose rotary table has {target.max_pos}")
    if temperature > 0:
        u = torch.as_tensor([] if u is None else u, dtype=torch.float32)
        if u.dim() != 2 or u.shape[0] < B or u.shape[1] < n_new:
            raise ValueError(f"expected uniforms [{B}][{n_new}] at least, got {list(u.shape)}")
    keep_first = min(keep_first, budget)
    keep_recent = min(keep_recent or (budget - keep_first) // 2, budget - keep_first)
    limit = budget + page_size                                        # where a sequence is brought back to its budget
    chunk = min(16, page_size, target.max_rows)
    pages = -(-limit // page_size)
    cache = PagedCache(target, B, B * pages, page_size, pages)
    everybody = range(B)
    evictions = used = 0

    def forward(kv, members, tokens, M, logits):
        """A pass over M rows of the sequences that kv holds, behind the eviction that makes room for them."""
        nonlocal evictions, used
        longest = max(cache.lengths[b] for b in members)
        if longest + M > limit:
            ss_paged_evict(kv, budget, keep_first=keep_first, keep_recent=keep_recent, max_len=longest)
            for b in members:
                cache.resize(b, min(cache.lengths[b], budget))
            evictions += 1
        for b in members:
            cache.resize(b, cache.lengths[b] + M)
        used = max(used, sum(len(p) for p in cache.pages))
        return ss_paged_forward(target, kv, tokens, M, logits=logits, weights=True, max_len=max(cache.lengths[b] for b in members))

    for b, prompt in enumerate(prompts):      # prompts of different lengths: all but the last token, sequence by sequence
        kv = cache.one(b)
        for i in range(0, len(prompt) - 1, chunk):
            part = torch.tensor([list(prompt[i:min(i + chunk, len(prompt) - 1)])], dtype=torch.int32, device=dev)
            forward(kv, [b], part, part.shape[1], False)
    tokens = torch.empty((n_new + 1, B), dtype=torch.int32, device=dev)
    tokens[0] = torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device=dev)
    logits = torch.empty((B, 1, V), dtype=torch.float32, device=dev)
    none = torch.empty(B, dtype=torch.int32, device=dev)
    uniforms = u.to(dev) if temperature > 0 else None
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for i in range(n_new):
        forward(cache.kv, everybody, tokens[i].view(B, 1), 1, logits)
        if temperature == 0:
            ss_greedy_accept(logits, None, none, tokens[i + 1])       # no draft tokens: the argmax
        else:
            ss_speculative_accept(ss_softmax(logits, temperature), None, None, uniforms[:, i:i + 1].contiguous(), none, tokens[i + 1])
    torch.cuda.synchronize()
    if stats is not None:
        stats.update(evictions=evictions, pages=used, loop_seconds=time.perf_counter() - t0)
    if int(cache.kv.status[0]):
        raise SpecVerifyError(-1, f"cache status {int(cache.kv.status[0])} after a decode loop (bit 3: a page that does not exist, bit 4: a length cut)")
    return [tokens[1:, b].tolist() for b in range(B)]
