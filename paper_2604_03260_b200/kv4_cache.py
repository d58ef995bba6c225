"""The 4-bit cache of one attention layer as a serving loop keeps it: a pool of pages, and for each of a fixed number of sequences
the pages that hold its tokens.

Pages, page table and lengths are on the GPU (``binding.make_kv4``); which pages are free, and how many sequences share a page, is host
bookkeeping.  The entry points that it calls are those of the C ABI (through ``binding``):

    append    focus_kv4_append, after the pages for the new tokens are found (and the page that a sequence is about to write to is
              copied, focus_kv4_copy_pages, if another sequence shares it)
    decode    focus_kv4_decode_step, one new query per sequence
    read      focus_kv4_read, tokens back in bf16 (focus_attn_fwd goes over a prefix with the queries of all its tokens)
    fork      another sequence with the same tokens: pages are shared, none is copied yet
    free      a sequence is forgotten; pages that no other sequence shares are free again
    compact   pages in use move to the front of the pool (focus_kv4_copy_pages)

A call whose pages do not fit raises ``FocusError`` (capacity), one whose tensors are refused what ``binding`` raises.  No call that
raises, wherever on its way, changes what the sequences hold.  All calls enqueue on the current stream (or ``stream``); use one
stream, or order them.  Sequences without tokens take part in ``decode`` with o = 0.

``decode`` and ``read`` only enqueue, as the entry points do.  ``append``, ``reserve``, ``fork``, ``free`` and ``compact`` cannot be
captured into a graph: they write the whole page table and all lengths anew on the host and copy them from pageable memory, and the host
waits until the stream has come to that copy.  Besides the wait a call takes 0.2 ms for one sequence of 130000 tokens in pages of 64,
0.4 ms for 32 of 5000 and 1.5 ms for 128 of 5000.  A loop for which that is too long keeps a table and lengths of its own and calls
``focus_kv4_append``.
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as fb


class Kv4Cache:
    """``sequences`` rows of at most ``max_tokens`` tokens over ``num_pages`` pages of ``page_tokens``; the other arguments as in
    ``binding.make_shape`` and ``binding.make_kv4``."""

    def __init__(self, sequences, Hq, Hkv, D, K, topk, window, max_tokens, num_pages, page_tokens=64, scale=0.0, softcap=0.0, k_scale=1.0, v_scale=1.0,
                 device="cuda"):
        self.B, self.Hkv, self.P = sequences, Hkv, page_tokens
        self._args = (Hq, Hkv, D, K, topk, window, scale, softcap)
        self.shape = self._shape(max_tokens)
        page_bytes = fb.focus_kv4_page_bytes(self.shape, page_tokens)
        if page_bytes == 0:
            raise fb.FocusError(-1, fb.lib().focus_last_error().decode())
        self.per_seq = -(-max_tokens // page_tokens)
        self.max_tokens, self.device = max_tokens, device
        self.pages = torch.zeros((num_pages, page_bytes), dtype=torch.uint8, device=device)
        self.book = torch.zeros(sequences * (self.per_seq + 1), dtype=torch.int32, device=device)       # page table and lengths, copied as one
        self.table, self.lens = self._parts(self.book)
        self.status = torch.zeros(4, dtype=torch.int32, device=device)
        self.ws = torch.empty(fb.focus_kv4_decode_workspace_bytes(self.shape), dtype=torch.uint8, device=device)
        self.cache = fb.make_kv4(self.pages, page_tokens, self.table, self.lens, k_scale, v_scale) if self.pages.is_cuda else None
        self.refs = [0] * num_pages                        # sequences that share a page; 0 = free
        self.held = [[] for _ in range(sequences)]         # the pages of a sequence, in order
        self.tokens = [0] * sequences
        self.stale = False                                 # the GPU may have another book than this (a copy of it failed): the next call brings it there

    def _shape(self, n):
        Hq, Hkv, D, K, topk, window, scale, softcap = self._args
        return fb.make_shape(Hq, Hkv, n, D, K, topk, window, scale, softcap, batch=self.B)

    def _parts(self, book):
        """page table and lengths of a book"""
        return book[:self.B * self.per_seq].view(self.B, self.per_seq), book[self.B * self.per_seq:]

    def _push(self, stream=None):
        """page table and lengths to the GPU, in one copy: both or neither"""
        book = torch.zeros(self.book.shape, dtype=torch.int32)
        table, lens = self._parts(book)
        for b, pages in enumerate(self.held):
            table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        lens[:] = torch.tensor(self.tokens, dtype=torch.int32)
        self.stale = True
        with torch.cuda.stream(stream):
            self.book.copy_(book)
        self.stale = False

    @contextlib.contextmanager
    def _or_as_before(self):
        """What fails inside leaves pages and tokens as they were.  Inside, they are replaced, not written to, and pages are copied into free ones alone,
        so that the book on the GPU stays right until the new one is there."""
        before = self.refs, self.held, self.tokens
        try:
            yield
        except BaseException:
            self.refs, self.held, self.tokens = before
            raise

    def _move(self, pairs, stream=None):
        if not pairs:
            return
        with torch.cuda.stream(stream):
            lists = torch.tensor(pairs, dtype=torch.int32).t().contiguous().to(self.device)
        fb.focus_kv4_copy_pages(self.shape, self.cache, lists[0], lists[1], self.status, stream)
        if stream is not None:
            lists.record_stream(stream)

    def plan(self, counts):
        """what ``counts`` new tokens of every sequence need: (pages of the sequences afterwards, pages to copy [(from, to)]).  Changes nothing."""
        if len(counts) != self.B or min(counts) < 0:
            raise fb.FocusError(-1, "one count >= 0 per sequence is wanted")
        refs, held, copies = list(self.refs), [list(p) for p in self.held], []
        free = (p for p, r in enumerate(self.refs) if r == 0)           # lowest first
        for b, c in enumerate(counts):
            if c == 0:
                continue
            if self.tokens[b] + c > self.max_tokens:
                raise fb.FocusError(-3, f"sequence {b}: {self.tokens[b]} + {c} tokens, at most {self.max_tokens}")
            need = -(-(self.tokens[b] + c) // self.P)
            take = [next(free, None) for _ in range(need - len(held[b]))]
            if self.tokens[b] % self.P and refs[held[b][-1]] > 1:         # the page it writes to next is another's too
                last = held[b].pop()
                refs[last] -= 1
                own = next(free, None)
                copies.append((last, own))
                take.insert(0, own)
            if None in take:
                raise fb.FocusError(-3, f"the pool of {len(refs)} pages is used up")
            for p in take:
                refs[p] = 1
            held[b] += take
        return refs, held, copies

    def reserve(self, counts, stream=None):
        """Room for ``counts`` new tokens of every sequence, which count as its last ones from here on."""
        refs, held, copies = self.plan(counts)
        with self._or_as_before():
            self.refs, self.held = refs, held
            self.tokens = [t + c for t, c in zip(self.tokens, counts)]
            self._move(copies, stream)
            self._push(stream)

    def append(self, k, v, mk, counts=None, stream=None):
        """k, v bf16 [sequences, Hkv, n, D], mk int32 [sequences*Hkv, n]: the first ``counts[b]`` tokens of every sequence (None: all n)"""
        n = k.shape[2]
        each = [n] * self.B if counts is None else list(counts)
        if len(each) != self.B or max(each) > n:
            raise fb.FocusError(-1, f"one count of at most {n} per sequence is wanted")
        reserved = False
        try:
            with self._or_as_before():
                self.reserve(each, stream)
                reserved = True
                with torch.cuda.stream(stream):
                    dev = None if counts is None else torch.tensor(each, dtype=torch.int32).to(self.device)
                fb.focus_kv4_append(self._shape(n), self.cache, k, v, mk, dev, self.status, stream)
        except BaseException:                              # refused: nothing is written, and the tokens do not count
            if reserved:
                self.stale = True                          # (should this fail too)
                self._push(stream)
            raise
        if dev is not None and stream is not None:
            dev.record_stream(stream)

    def decode(self, q, mq_new, o, lse, stream=None):
        """q, o bf16 [sequences, Hq, D]; the newest token of every sequence, appended before, is the query"""
        if self.stale:
            self._push(stream)
        fb.focus_kv4_decode_step(self.shape, self.cache, q, mq_new, o, lse, self.ws, self.status, stream)

    def read(self, k, v, mk=None, first=None, stream=None):
        """tokens first[b] .. first[b] + n - 1 of every sequence into k, v bf16 [sequences, Hkv, n, D]; rows behind the last token stay"""
        if self.stale:
            self._push(stream)
        fb.focus_kv4_read(self._shape(k.shape[2]), self.cache, first, k, v, mk, self.status, stream)

    def fork(self, source, target, stream=None):
        """sequence ``target``, which must be empty, gets the tokens of ``source``"""
        if source == target or self.tokens[target]:
            raise fb.FocusError(-1, f"sequence {target} is not empty")
        with self._or_as_before():
            self.refs, self.held, self.tokens = list(self.refs), list(self.held), list(self.tokens)
            for p in self.held[source]:
                self.refs[p] += 1
            self.held[target], self.tokens[target] = list(self.held[source]), self.tokens[source]
            self._push(stream)

    def free(self, sequence, stream=None):
        with self._or_as_before():
            self.refs, self.held, self.tokens = list(self.refs), list(self.held), list(self.tokens)
            for p in self.held[sequence]:
                self.refs[p] -= 1
            self.held[sequence], self.tokens[sequence] = [], 0
            self._push(stream)

    def compact(self, stream=None):
        """Pages in use to the front of the pool; the number of pages in use.  Sources lie behind it and targets before, so no page is both."""
        used = sum(r > 0 for r in self.refs)
        holes = [p for p in range(used) if self.refs[p] == 0]
        late = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(late, holes))
        with self._or_as_before():
            self.refs = list(self.refs)
            for a, z in to.items():
                self.refs[z], self.refs[a] = self.refs[a], 0
            self.held = [[to.get(p, p) for p in pages] for pages in self.held]
            self._move(list(to.items()), stream)
            self._push(stream)
        return used
