"""A paged cache of keys and values for LongNetAttention.step: pools of pages on
the GPU for every layer, one page table for all of them, kept on the host."""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple, Sequence

import torch


def xpos_span(gamma: float, scale_base: float) -> int:
    """How far from the xPos centre a position may lie: its scale is at most 2^64
    or at least 2^-64 there (dilated_attn_xpos, which takes the parameters in
    float32)."""
    gamma, scale_base = ctypes.c_float(gamma).value, ctypes.c_float(scale_base).value
    if not (0.0 < gamma < math.inf and 0.0 < scale_base < math.inf):
        raise ValueError("xPos needs a positive gamma and scale base")
    per = abs(math.log2(gamma / (1.0 + gamma)))
    span = int(64.0 * scale_base / per) + 1
    while span / scale_base * per > 64.0:
        span -= 1
    return span


@functools.lru_cache(maxsize=256)
def check_xpos(reach: int, center: int, gamma: float, scale_base: float):
    """Refuse a table of `reach` positions that xPos centred at `center` does not span."""
    span = xpos_span(gamma, scale_base)
    if not 0 <= center < reach or max(center, reach - 1 - center) > span:
        raise ValueError(f"xPos with gamma {gamma} and scale base {scale_base} spans {span} positions to each side of "
                         f"its centre, {2 * span + 1} positions in all: a table of {reach} with its centre at {center} "
                         f"does not fit")


class Batch(NamedTuple):
    """The sequences of one step, as cache_append and paged_attn take them:
    int32 device tensors [B, max_pages], [B] and [B + 1], and the most new
    tokens of a sequence; and all the new tokens (None: not known), the sequences
    with their new tokens, and the cache's number of the step."""
    block_table: torch.Tensor
    seq_lens: torch.Tensor
    q_start: torch.Tensor
    max_new: int
    tokens: int | None = None
    sequences: tuple = ()
    new: tuple = ()
    number: int = 0


class PagedCache:
    """Pages of page_size tokens (a power of two) for `layers` attention layers.

    k and v are lists with a tensor [num_pages, num_heads, page_size, head_dim]
    per layer; page p of every layer belongs to the same sequence.  A sequence
    holds at most max_pages pages.  `center` is the xPos centre of every
    position (the middle of the reach by default), fixed for the cache's life.

    Layers with xPos serve sequences of at most 2 xpos_span(gamma, scale_base) + 1
    positions (36261 with their defaults), and the whole table has to fit.  xpos,
    the layers' (gamma, scale_base), checks that here; otherwise their first step
    refuses.
    """

    def __init__(self, num_pages: int, page_size: int, max_pages: int, num_heads: int, head_dim: int,
                 layers: int = 1, center: int | None = None, device=None, dtype=torch.bfloat16,
                 xpos: tuple | None = None):
        if page_size < 1 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two")
        if num_pages < 1 or max_pages < 1 or layers < 1:
            raise ValueError("num_pages, max_pages and layers must be at least 1")
        self.center = max_pages * page_size // 2 if center is None else center
        if xpos is not None:
            check_xpos(max_pages * page_size, self.center, *xpos)
        shape = (num_pages, num_heads, page_size, head_dim)
        self.k = [torch.empty(shape, device=device, dtype=dtype) for _ in range(layers)]
        self.v = [torch.empty(shape, device=device, dtype=dtype) for _ in range(layers)]
        self.page_size, self.max_pages = page_size, max_pages
        self.device = self.k[0].device
        self._free = list(range(num_pages - 1, -1, -1))
        self._pages: dict = {}
        self._length: dict = {}
        self._last: dict = {}  # the step in which a sequence was last extended
        self._number = 0

    def length(self, sequence) -> int:
        """Tokens that the cache holds of a sequence (any hashable name)."""
        return self._length.get(sequence, 0)

    def release(self, sequence):
        """Forget a sequence; its pages go back to the pool."""
        self._free += self._pages.pop(sequence, [])
        self._length.pop(sequence, None)
        self._last.pop(sequence, None)

    def retract(self, batch: Batch):
        """Take back the extend that gave this batch: its sequences have their
        earlier lengths again, and pages taken for it go back to the pool.  Only
        while no other extend of one of them, nor a release, came since."""
        if not batch.sequences or any(self._last.get(s) != batch.number for s in batch.sequences):
            raise ValueError("not the last batch of all its sequences")
        for s, n in zip(batch.sequences, batch.new):
            self._length[s] -= n
            pages, keep = self._pages[s], -(-self._length[s] // self.page_size)
            self._free += reversed(pages[keep:])
            del pages[keep:], self._last[s]
            if self._length[s] == 0:
                self.release(s)

    def extend(self, sequences: Sequence, new: Sequence[int]) -> Batch:
        """Room for `new` more tokens of each sequence (named for the first time,
        it is empty), and the batch of a step in which they come.  Every layer
        then takes this batch once; if a layer does not (it raises, say), the
        batch has to be taken back, or the next one attends to tokens that are
        not there."""
        if len(set(sequences)) != len(sequences) or len(new) != len(sequences) or not len(new):
            raise ValueError("sequences must be different ones, with a number of new tokens each")
        if min(new) < 0:
            raise ValueError("the numbers of new tokens must not be negative")
        lengths = [self.length(s) + n for s, n in zip(sequences, new)]
        need = [-(-n // self.page_size) for n in lengths]
        short = [n - len(self._pages.get(s, ())) for s, n in zip(sequences, need)]
        if max(need) > self.max_pages:
            raise ValueError(f"a sequence of {max(lengths)} tokens is beyond {self.max_pages} pages of {self.page_size}")
        if sum(short) > len(self._free):
            raise RuntimeError(f"{sum(short)} pages are needed and {len(self._free)} are free")
        self._number += 1
        table = torch.zeros((len(need), self.max_pages), dtype=torch.int32)
        for i, (s, n, more) in enumerate(zip(sequences, lengths, short)):
            pages = self._pages.setdefault(s, [])
            pages += [self._free.pop() for _ in range(more)]
            self._length[s], self._last[s] = n, self._number
            table[i, : len(pages)] = torch.tensor(pages, dtype=torch.int32)
        start = torch.zeros(len(need) + 1, dtype=torch.int32)
        start[1:] = torch.tensor(new, dtype=torch.int32).cumsum(0)
        lens = torch.tensor(lengths, dtype=torch.int32)
        return Batch(table.to(self.device), lens.to(self.device), start.to(self.device), max(new), sum(new),
                     tuple(sequences), tuple(new), self._number)
