"""Keys of one split that are looked up in several chunks, against float64 with bars
that one misplaced tile passes (paged_rows).

A workgroup of single tokens looks up the cache rows of 1024 keys at a time, one of
tiles those of 4096; a plan leaves that many keys to a split only where there are
many workgroups.  How many splits a plan makes follows from its workspace, and the
tests hold it to what they need."""
import numpy as np
import pytest
import torch

from tests.gpu_util import note, require_gpu, to64
from tests.paged_rows import row
from tests.test_paged_gpu import setup

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
PAPER = [(2048, 1), (4096, 2), (8192, 4), (16384, 6), (32768, 12)]
DENSE = [(1 << 20, 1)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def check_rows(q, out, lse, seqs, lens, start, new, patterns, rows, group, tag):
    """rows: (sequence, its i-th new token, head)."""
    o64, l64 = to64(out), to64(lse)
    known = {}
    for b, i, h in rows:
        if (b, h // group) not in known:
            known[b, h // group] = [to64(t[:, h // group]) for t in seqs[b]]
        k, v = known[b, h // group]
        tok, pos = int(start[b]) + i, int(lens[b]) - new[b] + i
        ro, rl, bar = row(to64(q[tok, h]), k, v, pos, h, patterns)
        if np.isneginf(rl):
            assert np.isneginf(l64[h, tok]) and (o64[tok, h] == 0).all(), (tag, b, i, h)
            continue
        err = np.abs(o64[tok, h] - ro)
        assert (err <= bar).all(), f"{tag} {(b, i, h)}: {(err / bar).max():.2f} of the bar"
        assert abs(l64[h, tok] - rl) <= 1e-4, (tag, b, i, h)


def workspace(singles, one_slots, T, tile_slots, H, D):
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    one, tile = singles * H * one_slots, T * H * tile_slots
    return up(one * 4) + up(one * D * 4) + up(tile * 8) + up(tile * D * 2)


ONE = [
    # (cached before, H, Hkv, D, page, patterns, slots of a token)
    ([5000, 3333, 2048, 2047, 1024, 1025, 2080, 4200] + [3] * 56, 48, 48, 64, 64, DENSE, 1),
    ([4100, 2110, 3072, 1055] + [7] * 60, 192, 48, 128, 16, DENSE, 1),   # four query heads to a key head
    ([3000, 9000, 1300] + [0] * 61, 48, 48, 32, 8, DENSE, 1),
    ([32767, 30001, 29000, 32700] + [40] * 60, 12, 12, 64, 64, PAPER, 10),  # two splits of up to 1376 keys
]


@pytest.mark.parametrize("case", ONE, ids=lambda c: str(c[1:])[:50])
def test_single_tokens_of_many_chunks(case):
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    before, H, Hkv, D, page, patterns, slots = case
    note(f"[paged long] {case}")
    new = [1] * len(before)
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    T = len(new)
    need = paged_workspace_bytes(T, T, H, Hkv, D, kc.shape[0], page, dev[0].shape[1], patterns, 1)
    assert need == workspace(T, slots, 0, 0, H, D)
    out, lse = paged_attn(q, kc, vc, *dev, patterns, max_new=1)
    long = [b for b in range(T) if before[b] > 1000]
    rows = [(b, 0, h) for b in long for h in range(0, H, max(1, H // 12))] + [(T - 1, 0, 0), (T - 1, 0, H - 1)]
    check_rows(q, out, lse, seqs, lens, start, new, patterns, rows, H // Hkv, "single")


MANY = [
    # (new tokens, cached before, H, Hkv, D, page, patterns, splits of a tile's row)
    ([2200], [3000], 64, 2, 64, 64, DENSE, 1),
    ([2200], [6600], 64, 1, 128, 128, DENSE, 1),                       # three chunks
    ([2200], [6300], 64, 4, 32, 16, [(1 << 20, 1), (1 << 20, 2)], 2),  # 8500 and 4250 keys
    ([1200, 1100], [4500, 3100], 64, 2, 64, 32, DENSE, 1),
]


@pytest.mark.parametrize("case", MANY, ids=lambda c: str(c)[:50])
def test_tiles_of_many_chunks(case):
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    new, before, H, Hkv, D, page, patterns, slots = case
    note(f"[paged long] {case}")
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    T, B = sum(new), len(new)
    need = paged_workspace_bytes(T, B, H, Hkv, D, kc.shape[0], page, dev[0].shape[1], patterns, max(new))
    assert any(need == workspace(4 * B if B > 1 else 0, one, T, slots, H, D) for one in range(65))
    out, lse = paged_attn(q, kc, vc, *dev, patterns, max_new=max(new))
    rng = np.random.default_rng(1)
    rows = []
    for b in range(B):
        # around the chunks' ends, the first and last rows, and some in between
        at = [p - before[b] + d for p in range(4096, int(lens[b]) + 1, 4096) for d in (-1, 0, 1, 63, 64, 65)]
        at += [0, 1, 127, 128, new[b] - 1, new[b] - 2] + rng.integers(0, new[b], 12).tolist()
        rows += [(b, i, int(rng.integers(0, H))) for i in at if 0 <= i < new[b]]
    assert len(rows) > 12
    check_rows(q, out, lse, seqs, lens, start, new, patterns, rows, H // Hkv, "tiles")


def test_single_tokens_of_many_chunks_beside_tiles():
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    note("[paged long] beside tiles")
    H, D, page = 24, 64, 16
    new, before = [1] * 30 + [300] + [1] * 33, [3000, 2049, 1100] + [5] * 27 + [2500] + [9] * 30 + [4097, 1040, 2222]
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, H, D, page, BF)
    need = paged_workspace_bytes(sum(new), 64, H, H, D, kc.shape[0], page, dev[0].shape[1], DENSE, 300)
    tile_slots = next(s for s in range(1, 17) if need == workspace(256, 1, sum(new), s, H, D))  # a token's: one
    note(f"  {tile_slots} splits of the tiles' keys")
    out, lse = paged_attn(q, kc, vc, *dev, DENSE, max_new=300)
    rows = [(b, 0, h) for b in (0, 1, 2, 61, 62, 63, 10) for h in range(0, H, 3)]
    rows += [(30, i, h) for i in (0, 1, 150, 298, 299) for h in (0, 7, 23)]
    check_rows(q, out, lse, seqs, lens, start, new, DENSE, rows, 1, "beside tiles")


ALL = [
    # the same bars where keys are split, patterns overlap and rows meet in the join
    ([1], [4095], 12, 12, 64, 64, PAPER),
    ([1, 1], [1500, 2600], 8, 2, 128, 32, DENSE),
    ([70], [4500], 2, 1, 128, 128, DENSE),
    ([100], [1500], 3, 3, 64, 16, [(2048, 1), (2048, 2), (4096, 1), (1024, 1), (3000, 2), (5000, 3)]),
    ([60, 1, 1], [1200, 3000, 40], 4, 2, 128, 32, [(512, 1), (4096, 1)]),
    ([300, 1, 2], [2000, 3500, 1], 6, 6, 32, 8, [(4096, 1), (1024, 3)]),
    ([512], [8000], 12, 12, 64, 64, PAPER),
]


@pytest.mark.parametrize("case", ALL, ids=lambda c: str(c)[:50])
def test_rows_within_their_own_error(case):
    from paper_2307_02486_amd import paged_attn
    new, before, H, Hkv, D, page, patterns = case
    note(f"[paged long] {case}")
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    out, lse = paged_attn(q, kc, vc, *dev, patterns, max_new=max(new))
    rng = np.random.default_rng(2)
    rows = [(b, i, h) for b, n in enumerate(new) for i in sorted({0, n // 2, n - 1, *rng.integers(0, n, 8).tolist()})
            for h in range(H)]
    check_rows(q, out, lse, seqs, lens, start, new, patterns, rows, H // Hkv, "all")
