"""Values that are not finite in the cache: the rows that see their keys are not finite in
their elements, and nothing else is, whatever tile holds them.

Bars: those of test_paged8_gpu and test_paged_gpu, 5e-3 max|v| of the finite ones."""
import numpy as np
import pytest
import torch

from oracle.compressed_ref import attention_ref
from tests.cache8 import rows_of
from tests.gpu_util import note, require_gpu, to64
from tests.test_paged8_gpu import held_values
from tests.test_paged8_gpu import setup as setup8
from tests.test_paged_gpu import setup

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
PATS = [(64, 1), (256, 2), (512, 5)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def places(lens, new, Hkv, D):
    """(sequence, position, key head, element): cached ones, and new tokens that earlier
    new tokens of their tile do not see (the very last among them)."""
    out = []
    for b, n in enumerate(lens):
        for j, pos in enumerate((n - 1, n - 1 - new[b] // 3, n - 1 - new[b] // 2, n - new[b] - 3)):
            if pos >= 0:
                out.append((b, pos, (b + j) % Hkv, (7 * j + 5 * b + 3) % D))
    return out


def check(out, lse, q, seqs, theres, lens, start, patterns, tag):
    o64, l64, q64 = to64(out), to64(lse).T, to64(q)
    hit = other = 0
    for b, (k, v) in enumerate(seqs):
        rows, n = slice(start[b], start[b + 1]), int(start[b + 1] - start[b])
        with np.errstate(invalid="ignore"):
            want, wl = attention_ref(q64[rows], k, v, int(lens[b]) - n, patterns, theres[b])
        top = np.abs(v[np.isfinite(v)]).max()
        fin = np.isfinite(want)
        assert np.array_equal(np.isfinite(o64[rows]), fin), (tag, b)  # (zero times an infinite one is NaN)
        assert np.abs(o64[rows][fin] - want[fin]).max() <= 5e-3 * top, (tag, b)
        live = np.isfinite(wl)
        assert np.array_equal(live, np.isfinite(l64[rows])), (tag, b)
        assert np.abs(l64[rows][live] - wl[live]).max() <= 1e-4, (tag, b)
        hit, other = hit + int((~fin).sum()), other + int((fin & (~fin).any(0)).sum())  # the same element, earlier
    assert hit and (other or len(o64) < 16)  # a few rows may see all of them


NEW = [([70], [50]), ([300], [700]), ([3, 150], [200, 0]), ([1, 2], [90, 40]), ([1] * 20 + [200], [64] * 20 + [33])]


@pytest.mark.parametrize("D, H, Hkv, page", [(64, 4, 4, 16), (128, 4, 2, 64), (32, 6, 2, 8)], ids=str)
@pytest.mark.parametrize("new, before", NEW, ids=lambda x: str(x)[:20])
@pytest.mark.parametrize("gone", [0.0, 0.3], ids=str)
def test_a_cache_in_8_bits(D, H, Hkv, page, new, before, gone):
    from paper_2307_02486_amd import paged_attn
    note(f"[paged8] bad values D={D} {new} {gone}")
    q, kc, vc, ks, vs, dev, table, lens, start = setup8(new, before, H, Hkv, D, page, BF, gone)
    held = held_values(kc, vc, ks, vs)
    for b, pos, h, d in places(lens, new, Hkv, D):
        p = int(table[b, pos // page])
        if 0 <= p < kc.shape[0]:
            vc.view(torch.uint8)[p, h, pos % page, d] = 0x7F if pos % 2 else 0xFF
            held[1][p, h, pos % page, d] = np.nan
    out, lse = paged_attn(q, kc, vc, *dev, PATS, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    seqs, theres = [], []
    for b, n in enumerate(lens):
        k, there = rows_of(held[0], table[b], page, int(n))
        v, _ = rows_of(held[1], table[b], page, int(n))
        seqs.append((k, v))
        theres.append(there)
    check(out, lse, q, seqs, theres, lens, start, PATS, "8 bits")


@pytest.mark.parametrize("D, H, Hkv, page", [(64, 4, 4, 16), (128, 4, 2, 64), (32, 6, 2, 8)], ids=str)
@pytest.mark.parametrize("new, before", NEW, ids=lambda x: str(x)[:20])
@pytest.mark.parametrize("many", [False, True], ids=["5 patterns", "16 patterns"])
def test_a_wide_cache(D, H, Hkv, page, new, before, many):
    from paper_2307_02486_amd import paged_attn
    note(f"[paged] bad values D={D} {new}")
    pats = PATS + [(16 * i, i) for i in range(2, 9)] if many else PATS
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    for i, (b, pos, h, d) in enumerate(places(lens, new, Hkv, D)):
        v = seqs[b][1]
        v[pos, h, d] = (float("nan"), float("inf"), -float("inf"))[i % 3]
        vc[int(dev[0][b, pos // page]), h, pos % page] = v[pos, h]
    out, lse = paged_attn(q, kc, vc, *dev, pats)
    torch.cuda.synchronize()
    check(out, lse, q, [(to64(k), to64(v)) for k, v in seqs], [np.ones(int(n), bool) for n in lens], lens, start, pats,
          "wide")


LONG = [(4096, 1), (2048, 2)]  # keys in several splits, which lane groups of the join share


@pytest.mark.parametrize("D, H, Hkv, page", [(64, 4, 4, 64), (128, 2, 1, 16), (32, 3, 3, 128)], ids=str)
@pytest.mark.parametrize("eight", [True, False], ids=["8 bits", "wide"])
def test_rows_whose_keys_are_split(D, H, Hkv, page, eight):
    from paper_2307_02486_amd import paged_attn
    note(f"[paged] bad values in splits D={D} {eight}")
    new, before = [60], [3500]
    if eight:
        q, kc, vc, ks, vs, dev, table, lens, start = setup8(new, before, H, Hkv, D, page, BF, 0.3)
        held = held_values(kc, vc, ks, vs)
        for b, pos, h, d in places(lens, new, Hkv, D):
            p = int(table[b, pos // page])
            if 0 <= p < kc.shape[0]:
                vc.view(torch.uint8)[p, h, pos % page, d] = 0x7F
                held[1][p, h, pos % page, d] = np.nan
        out, lse = paged_attn(q, kc, vc, *dev, LONG, k_scale=ks, v_scale=vs)
        k, there = rows_of(held[0], table[0], page, int(lens[0]))
        v, _ = rows_of(held[1], table[0], page, int(lens[0]))
        check(out, lse, q, [(k, v)], [there], lens, start, LONG, "8 bits")
        return
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    for b, pos, h, d in places(lens, new, Hkv, D):
        v = seqs[b][1]
        v[pos, h, d] = float("nan")
        vc[int(dev[0][b, pos // page]), h, pos % page] = v[pos, h]
    out, lse = paged_attn(q, kc, vc, *dev, LONG)
    check(out, lse, q, [(to64(k), to64(v)) for k, v in seqs], [np.ones(int(n), bool) for n in lens], lens, start, LONG,
          "wide")
