"""A paged cache of keys and values for LongNetAttention.step: pools of pages on
the GPU for every layer, one page table for all of them, kept on the host."""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple, Sequence

import torch

from .ops import CACHE_BLOCK, CACHE_F8, CACHE_SCALE, cache_scale_shape, evict_pages


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

    dtype float8_e4m3fn makes a cache in 8 bits, whose scales are the lists k_scale
    and v_scale.  With weigh=True it counts in `weights` (float32 [num_pages]) the
    attention that its pages get in each step, all layers together, and `evict` gives
    up the pages that got least.  Pages of a sequence that are gone are -1 in its
    table; its tokens keep their positions.
    """

    def __init__(self, num_pages: int, page_size: int, max_pages: int, num_heads: int, head_dim: int,
                 layers: int = 1, center: int | None = None, device=None, dtype=torch.bfloat16,
                 xpos: tuple | None = None, weigh: bool = False):
        if page_size < 1 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two")
        if num_pages < 1 or max_pages < 1 or layers < 1:
            raise ValueError("num_pages, max_pages and layers must be at least 1")
        self.center = max_pages * page_size // 2 if center is None else center
        if xpos is not None:
            check_xpos(max_pages * page_size, self.center, *xpos)
        if weigh and dtype != CACHE_F8:
            raise ValueError(f"weigh goes with a cache of {CACHE_F8}")
        shape = (num_pages, num_heads, page_size, head_dim)
        self.k_scale = self.v_scale = self.weights = None
        self._blocks = []  # 8 bits: bytes of k, k_scale, v, v_scale [layers, num_pages, num_heads, blocks of a page, ...]
        with torch.inference_mode(False):  # extend and retract write them in any mode
            if dtype == CACHE_F8:
                self.k, self.k_scale, self.v, self.v_scale = (self._pool(layers, *x, device) for x in (
                    (shape, dtype), (cache_scale_shape(shape), CACHE_SCALE)) * 2)
            else:
                self.k = [torch.empty(shape, device=device, dtype=dtype) for _ in range(layers)]
                self.v = [torch.empty(shape, device=device, dtype=dtype) for _ in range(layers)]
            if weigh:
                self.weights = torch.zeros(num_pages, device=device)
        self.page_size, self.max_pages = page_size, max_pages
        self.device = self.k[0].device
        self._free = list(range(num_pages - 1, -1, -1))
        self._pages: dict = {}
        self._length: dict = {}
        self._last: dict = {}  # the step in which a sequence was last extended
        self._before: dict = {}  # 8 bits: by step, the blocks that its tokens share with earlier ones, as they were
        self._number = 0

    def _pool(self, layers: int, shape: tuple, dtype, device) -> list:
        """A tensor of this shape for each layer, of one allocation."""
        pool = torch.empty((layers, *shape), device=device, dtype=dtype)
        self._blocks.append(pool.view(torch.uint8).view(layers, *shape[:2], shape[2] // min(shape[2], CACHE_BLOCK), -1)
                            if len(shape) == 4 else pool.view(torch.uint8))
        return list(pool.unbind(0))

    def length(self, sequence) -> int:
        """Tokens that the cache holds of a sequence (any hashable name)."""
        return self._length.get(sequence, 0)

    def release(self, sequence):
        """Forget a sequence; its pages go back to the pool."""
        self._free += [p for p in self._pages.pop(sequence, []) if p >= 0]
        self._length.pop(sequence, None)
        self._settle(sequence)

    def _settle(self, sequence):
        """The sequence's last batch cannot be taken back any more."""
        self._before.pop(self._last.pop(sequence, None), None)

    def _keep_blocks(self, sequences: Sequence, new: Sequence[int]):
        """The blocks in which these new tokens follow earlier ones, as they are: their
        page and number in it, the earlier tokens, and their bytes.  An append may take a
        larger scale for such a block and round its earlier values once more."""
        size, at = min(self.page_size, CACHE_BLOCK), []
        for s, n in zip(sequences, new):
            had = self.length(s)
            page = self._pages[s][had // self.page_size] if n > 0 and had % size else -1
            if page >= 0:
                at.append((page, had % self.page_size // size, had % size))
        if not at:
            return None
        page, block, rows = torch.tensor(at).t().contiguous().to(self.device)
        return page, block, rows, [b[:, page, :, block] for b in self._blocks]

    def _put_back(self, page, block, rows, kept: list):
        """The blocks of _keep_blocks, where an append has rescaled them.  A block whose
        earlier values are not what rescaling makes of those kept (the batch before had not
        run when they were kept) stays as it is."""
        size = min(self.page_size, CACHE_BLOCK)
        for i in (0, 2):  # k and v, each with its scale
            was, scale = kept[i], kept[i + 1]
            now, now_scale = (b[:, page, :, block] for b in self._blocks[i: i + 2])
            more = now_scale.int() - scale.int()
            want = (was.view(CACHE_F8).double() * torch.exp2(-more.double())[..., None]).float().to(CACHE_F8).float()
            have = now.view(CACHE_F8).float()
            same = ((want == have) | (want.isnan() & have.isnan())).view(*was.shape[:-1], size, -1).all(-1)
            earlier = torch.arange(size, device=rows.device) < rows[:, None]
            back = (same | ~earlier[:, None, None]).all(-1) & (more > 0)
            self._blocks[i][:, page, :, block] = torch.where(back[..., None], was, now)
            self._blocks[i + 1][:, page, :, block] = torch.where(back, scale, now_scale)

    def retract(self, batch: Batch):
        """Take back the extend that gave this batch: its sequences have their
        earlier lengths again, and pages taken for it go back to the pool.  Only
        while no other extend of one of them, nor a release or an evict, came since.
        In a cache in 8 bits, blocks that its layers rescaled have their earlier values
        and scales again, if the batches before had run when it was made.  What its
        layers added to the weights of other pages stays."""
        if not batch.sequences or any(self._last.get(s) != batch.number for s in batch.sequences):
            raise ValueError("not the last batch of all its sequences")
        if kept := self._before.pop(batch.number, None):
            self._put_back(*kept)
        for s, n in zip(batch.sequences, batch.new):
            self._length[s] -= n
            pages, keep = self._pages[s], -(-self._length[s] // self.page_size)
            self._free += [p for p in reversed(pages[keep:]) if p >= 0]
            del pages[keep:], self._last[s]
            if self._length[s] == 0:
                self.release(s)

    def evict(self, keep: int, sequences: Sequence | None = None, first: int = 1, last: int = 1) -> int:
        """Give up the pages of least weight of each of these sequences (default:
        all), until it has `keep`; never its first `first` pages nor its last `last`
        (see evict_pages), of which the last takes the next tokens.  They go back to
        the pool.  Only between steps: a batch made before names them still.  Waits
        for the GPU.  Returns how many went."""
        if self.weights is None:
            raise ValueError("evict needs a cache that counts its pages' weights (weigh=True)")
        if keep < 0 or first < 0 or last < 1:
            raise ValueError("keep and first must not be negative, and last at least 1")
        names = list(self._pages if sequences is None else sequences)
        if len(set(names)) != len(names) or any(s not in self._pages for s in names):
            raise ValueError("sequences must be different ones that the cache holds")
        if not names:
            return 0
        lens = torch.tensor([self._length[s] for s in names], dtype=torch.int32).to(self.device)
        _, freed, count = evict_pages(self.weights, self._table(names).to(self.device), lens, self.page_size, keep,
                                      first, last)
        freed, count = freed.cpu(), count.tolist()
        for s, row, n in zip(names, freed, count):
            if n:
                gone = set(row[:n].tolist())
                self._pages[s] = [-1 if p in gone else p for p in self._pages[s]]
                self._free += reversed(sorted(gone))
                self._settle(s)  # a batch made before names pages that went
        return sum(count)

    def _table(self, names: Sequence) -> torch.Tensor:
        """The rows of these sequences in a table on the host."""
        table = torch.full((len(names), self.max_pages), -1 if self.k_scale is not None else 0, dtype=torch.int32)
        for i, s in enumerate(names):
            table[i, : len(self._pages[s])] = torch.tensor(self._pages[s], dtype=torch.int32)
        return table

    def extend(self, sequences: Sequence, new: Sequence[int]) -> Batch:
        """Room for `new` more tokens of each sequence (named for the first time,
        it is empty), and the batch of a step in which they come.  Every layer
        then takes this batch once; if a layer does not (it raises, say), the
        batch has to be taken back, or the next one attends to tokens that are
        not there.  For that a cache in 8 bits keeps the blocks of 16 tokens that the
        new ones share with earlier ones, until a sequence's next extend."""
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
        kept = self._keep_blocks(sequences, new) if self._blocks else None
        for s in sequences:
            self._settle(s)
        self._number += 1
        if kept is not None:
            self._before[self._number] = kept
        taken = []
        for s, n, more in zip(sequences, lengths, short):
            taken += (fresh := [self._free.pop() for _ in range(more)])
            self._pages.setdefault(s, []).extend(fresh)
            self._length[s], self._last[s] = n, self._number
        table = self._table(sequences)
        if self.weights is not None and taken:  # whoever had these pages before, they begin without weight
            self.weights[torch.tensor(taken, device=self.device)] = 0.0
        start = torch.zeros(len(need) + 1, dtype=torch.int32)
        start[1:] = torch.tensor(new, dtype=torch.int32).cumsum(0)
        lens = torch.tensor(lengths, dtype=torch.int32)
        return Batch(table.to(self.device), lens.to(self.device), start.to(self.device), max(new), sum(new),
                     tuple(sequences), tuple(new), self._number)
