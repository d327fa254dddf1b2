"""Dilated attention over a cache in 8 bits against float64, every row, on the
values that the cache holds; some pages are gone.

An element of the cache is exact in bf16 and float32, so the bars are those of
the attention over a cache of those types: bf16, |out - ref| <= 5e-3 max|v| and
|lse - ref| <= 1e-4; float32, 2e-5 max|v| and 1e-4."""
import numpy as np
import pytest
import torch

import workloads
from oracle.compressed_ref import attention_ref
from tests.cache8 import E8, F8, elements, normal_pool, rows_of
from tests.gpu_util import note, require_gpu, to64
from tests.paged_rows import row
from tests.test_heads_gpu import paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
PAPER = [(2048, 1), (4096, 2), (8192, 4), (16384, 6), (32768, 12)]
DENSE = [(1 << 20, 1)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def setup(new, before, H, Hkv, D, page, dtype, gone=0.3, seed=0):
    """Queries, caches and tables: whatever no sequence holds is NaN, pages that are
    gone are -1 or past the pool (a sequence's last one stays)."""
    table, lens, start, dev, pages = paged(new, before, page, seed=seed)
    rng = np.random.default_rng(seed + 5)
    for b, n in enumerate(lens):
        last = max(-(-int(n) // page) - 1, 0)
        out = np.flatnonzero(rng.random(last) < gone)
        table[b, out] = np.where(rng.random(len(out)) < 0.5, -1, 2 ** 30)
    dev[0].copy_(torch.from_numpy(table))
    q = workloads.make_random((max(int(start[-1]), 1), H, D), dtype, 1.0, 300 + seed, "cuda", 0)[: int(start[-1])]
    kc, ks = normal_pool(pages, Hkv, page, D, seed + 1)
    vc, vs = normal_pool(pages, Hkv, page, D, seed + 2)
    held = np.zeros((pages, page), bool)
    for b, n in enumerate(lens):
        at = np.arange(int(n))
        p = table[b, at // page]
        ok = (p >= 0) & (p < pages)
        held[p[ok], at[ok] % page] = True
    for c in (kc, vc):
        c.view(torch.uint8)[torch.from_numpy(~held).cuda()[:, None].expand(-1, Hkv, -1)] = 0x7F
    return q, kc, vc, ks, vs, dev, table, lens, start


def compare(out, lse, q, pools, table, lens, start, page, patterns, dtype, tag, scale=None):
    to, tl = (5e-3, 1e-4) if dtype == BF else (2e-5, 1e-4)
    out, lse, q64 = to64(out), to64(lse).T, to64(q)
    for b, n in enumerate(lens):
        rows = slice(start[b], start[b + 1])
        new = start[b + 1] - start[b]
        if new == 0:
            continue
        k, there = rows_of(pools[0], table[b], page, int(n))
        v, _ = rows_of(pools[1], table[b], page, int(n))
        ro, rl = attention_ref(q64[rows], k, v, n - new, patterns, there, scale)
        assert np.array_equal(np.isneginf(rl), np.isneginf(lse[rows])), f"{tag} {b}: rows without keys"
        assert not np.isnan(out[rows]).any() and not np.isnan(lse[rows]).any(), f"{tag} {b}: NaN"
        assert (out[rows][np.isneginf(rl)] == 0).all(), f"{tag} {b}: rows without keys are zero"
        eo = np.abs(out[rows] - ro).max() / max(np.abs(v).max(), 1e-30)
        fin = np.isfinite(rl)
        el = np.abs(lse[rows][fin] - rl[fin]).max() if fin.any() else 0.0
        assert eo <= to and el <= tl, f"{tag} {b}: out {eo:.2e} (bar {to}), lse {el:.2e} (bar {tl})"


def held_values(kc, vc, ks, vs):
    """The pools' elements, zero where NaN (no sequence's)."""
    return [np.nan_to_num(elements(c, s)) for c, s in ((kc, ks), (vc, vs))]


CASES = [
    # (new tokens, cached before, H, Hkv, D, page, patterns, dtype)
    ([1], [0], 1, 1, 64, 16, DENSE, BF),
    ([1], [4095], 12, 12, 64, 64, PAPER, BF),
    ([1, 1, 1], [0, 31, 700], 12, 12, 64, 16, [(64, 1), (256, 3), (1024, 5)], BF),
    ([1, 1], [1500, 2600], 8, 2, 128, 32, DENSE, BF),
    ([1, 4, 2], [300, 5, 77], 24, 1, 64, 8, [(128, 1), (512, 2)], BF),
    ([3, 3], [100, 1000], 6, 3, 32, 1, [(100, 1), (333, 7)], BF),
    ([1, 2], [63, 64], 8, 4, 64, 64, [(64, 2), (128, 3), (512, 9)], BF),
    ([2, 1], [40, 90], 5, 5, 64, 16, [(32, 1), (32, 1), (96, 1), (64, 2)], BF),
    ([5], [0], 4, 4, 64, 16, DENSE, BF),
    ([130], [0], 3, 3, 64, 16, [(64, 1), (128, 2)], BF),
    ([257], [1000], 4, 2, 64, 64, [(300, 1), (700, 3), (1 << 30, 11)], BF),
    ([70], [4500], 2, 1, 128, 128, DENSE, BF),                # more keys than are looked up at once
    ([300], [17], 6, 6, 32, 8, [(100, 2), (400, 5)], BF),     # rows without keys in tiles
    ([64, 1, 200, 0, 3], [10, 2000, 0, 50, 129], 12, 4, 64, 16, [(256, 1), (512, 2), (4096, 4)], BF),
    ([1] * 20 + [90] + [1] * 50, list(range(0, 710, 10)), 4, 4, 64, 32, [(128, 1), (512, 4)], BF),
    ([300] + [1] * 39, list(range(0, 400, 10)), 12, 12, 64, 16, [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)], BF),
    ([5, 4, 6, 1], [90, 80, 0, 7], 16, 4, 128, 16, [(64, 1), (4096, 2)], BF),
    ([1, 7, 40], [0, 600, 33], 6, 2, 32, 16, [(512, 1), (600, 3)], F32),
    ([3], [1000], 4, 4, 64, 64, DENSE, F32),
    ([1, 33], [300, 0], 4, 1, 128, 8, [(64, 2), (128, 3)], F32),
    ([40, 2], [40, 3], 3, 3, 64, 16, [(16, 1), (48, 1), (1 << 20, 2)] + [(8 * i, i) for i in range(2, 15)], BF),
    ([100], [1500], 3, 3, 64, 16, [(2048, 1), (2048, 2), (4096, 1), (1024, 1), (3000, 2), (5000, 3)], BF),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:60])
@pytest.mark.parametrize("gone", [0.0, 0.3, 1.0], ids=str)
def test_matches_the_definition(case, gone):
    from paper_2307_02486_amd import paged_attn
    new, before, H, Hkv, D, page, patterns, dtype = case
    note(f"[paged8] {gone} {str(case)[:200]}")
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, before, H, Hkv, D, page, dtype, gone)
    sc = dict(k_scale=ks, v_scale=vs)
    out, lse = paged_attn(q, kc, vc, *dev, patterns, **sc)
    hint = paged_attn(q, kc, vc, *dev, patterns, max_new=max(new), **sc)
    wrong = paged_attn(q, kc, vc, *dev, patterns, max_new=1, **sc)
    torch.cuda.synchronize()
    pools = held_values(kc, vc, ks, vs)
    compare(out, lse, q, pools, table, lens, start, page, patterns, dtype, "no hint")
    compare(*hint, q, pools, table, lens, start, page, patterns, dtype, "hint")
    compare(*wrong, q, pools, table, lens, start, page, patterns, dtype, "a hint of one whatever the lengths")
    again = paged_attn(q, kc, vc, *dev, patterns, **sc)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("D, dtype", [(32, BF), (64, BF), (128, BF), (64, F32)], ids=str)
@pytest.mark.parametrize("new", [[1, 1], [2, 90]], ids=str)
def test_is_the_attention_over_a_cache_of_the_same_values(D, dtype, new):
    """All pages there: within the rounding of sums of the attention over a wide
    cache that holds the same elements (bf16: out within two of its steps of the
    row's size, as probabilities and out are rounded alike from scores that differ by
    float32 sums in another order)."""
    from paper_2307_02486_amd import paged_attn
    note(f"[paged8] wide {D} {dtype} {new}")
    pats, page, H, Hkv = [(256, 1), (1000, 3)], 16, 6, 2
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [700, 333], H, Hkv, D, page, dtype, 0.0)
    wide = [torch.from_numpy(x).to(dtype).cuda() for x in held_values(kc, vc, ks, vs)]
    assert all(np.array_equal(to64(w), x) for w, x in zip(wide, held_values(kc, vc, ks, vs)))  # exact
    want, want_lse = paged_attn(q, *wide, *dev, pats)
    out, lse = paged_attn(q, kc, vc, *dev, pats, k_scale=ks, v_scale=vs)
    assert float((lse - want_lse).abs().max()) <= 2e-5
    bar = 2.0 ** -6 if dtype == BF else 2e-5
    assert float((out.float() - want.float()).abs().max()) <= bar * float(want.float().abs().max())


@pytest.mark.parametrize("spread", [1e-30, 1e-6, 1e5, 1e30], ids=str)
@pytest.mark.parametrize("new", [[1], [80]], ids=str)
def test_values_of_any_size(spread, new):
    """Scales of V far from one: outputs keep bf16's precision relative to V."""
    from paper_2307_02486_amd import paged_attn
    note(f"[paged8] values {spread} {new}")
    pats = [(128, 1), (512, 2)]
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [300], 4, 4, 64, 16, BF)
    more = int(np.rint(np.log2(spread)))
    vs = (vs.view(torch.uint8).to(torch.int32) + more).to(torch.uint8).view(E8)
    out, lse = paged_attn(q, kc, vc, *dev, pats, k_scale=ks, v_scale=vs)
    compare(out, lse, q, held_values(kc, vc, ks, vs), table, lens, start, 16, pats, BF, f"values {spread}")


@pytest.mark.parametrize("D, H, Hkv, page", [(64, 12, 12, 64), (128, 8, 2, 16), (32, 4, 4, 8)], ids=str)
@pytest.mark.parametrize("n", [1, 600], ids=str)
def test_long_sequences_row_by_row(D, H, Hkv, page, n):
    """Thousands of keys: sampled rows within bf16's own error in each element, so
    that a tile, a block's scale or a page in the wrong place shows."""
    from paper_2307_02486_amd import paged_attn
    note(f"[paged8] long D={D} n={n}")
    q, kc, vc, ks, vs, dev, table, lens, start = setup([n], [20000], H, Hkv, D, page, BF, 0.4)
    out, lse = paged_attn(q, kc, vc, *dev, PAPER, k_scale=ks, v_scale=vs, max_new=n)
    pools = held_values(kc, vc, ks, vs)
    L = int(lens[0])
    k, there = rows_of(pools[0], table[0], page, L)
    v, _ = rows_of(pools[1], table[0], page, L)
    rng = np.random.default_rng(4)
    for i in sorted({0, n - 1, *rng.integers(0, n, 6).tolist()}):
        for h in rng.permutation(H)[:3]:
            pos = 20000 + i
            kh, vh = k[:, h // (H // Hkv)], v[:, h // (H // Hkv)]
            # rows whose page is gone: out of the lists, by scores that weigh nothing
            kk = np.where(there[:, None], kh, 0.0)
            want, wl, bar = masked_row(to64(q)[i, h], kk, vh, pos, int(h), there)
            got = to64(out)[i, h]
            assert (np.abs(got - want) <= bar).all(), (i, h, float((np.abs(got - want) / bar).max()))
            assert np.isneginf(wl) == np.isneginf(float(lse[h, i])) and (np.isneginf(wl) or abs(float(lse[h, i]) - wl) <= 1e-4)


def masked_row(q, k, v, pos, head, there):
    """tests.paged_rows.row on the keys that are there, as a sequence of its own whose
    patterns hold a key as often as PAPER holds it."""
    from tests.paged_rows import key_counts
    c = key_counts(pos, k.shape[0], head, PAPER)[:, there[: k.shape[0]]]
    import tests.paged_rows as rows
    saved = rows.key_counts
    try:
        rows.key_counts = lambda *_: c
        return row(q, k[there], v[there], pos, head, PAPER)
    finally:
        rows.key_counts = saved


@pytest.mark.parametrize("new", [[1], [2, 90]], ids=str)
def test_strided_queries_given_outputs_and_scale(new):
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    note(f"[paged8] strided {new}")
    pats, H = [(64, 1), (256, 2)], 6
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [70, 5][: len(new)], H, 2, 64, 16, BF)
    T = q.shape[0]
    wide = torch.full((T, H + 5, 64), float("nan"), dtype=BF, device="cuda")
    wide[:, :H] = q
    out = torch.full((T, H, 64), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((H, T), float("nan"), device="cuda")
    need = paged_workspace_bytes(T, len(new), H, 2, 64, kc.shape[0], 16, dev[0].shape[1], pats)
    guard = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    got = paged_attn(wide[:, :H], kc, vc, *dev, pats, scale=0.3, out=out, lse=lse, workspace=guard[:need], k_scale=ks,
                     v_scale=vs)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse and bool((guard[need:] == 0x5A).all())
    compare(out, lse, q, held_values(kc, vc, ks, vs), table, lens, start, 16, pats, BF, "strided", 0.3)


def test_nan_keys_and_values_show_where_they_are_seen():
    """A NaN in a key's row is NaN in the rows that see it and nowhere else."""
    from paper_2307_02486_amd import paged_attn
    note("[paged8] NaN")
    for new in ([1, 1], [40, 1]):
        q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [50, 90], 4, 4, 64, 16, BF, 0.0)
        at = int(lens[0]) - 1  # the first sequence's last token
        kc.view(torch.uint8)[int(table[0, at // 16]), :, at % 16, 3] = 0x7F
        out, lse = paged_attn(q, kc, vc, *dev, DENSE, k_scale=ks, v_scale=vs)
        hit = new[0] - 1
        assert bool(torch.isnan(lse[:, hit]).all()) and bool(torch.isnan(out[hit].float()).all())
        rest = [t for t in range(sum(new)) if t != hit]
        assert bool(torch.isfinite(lse[:, rest]).all()) and bool(torch.isfinite(out[rest].float()).all())


def test_pool_beyond_4_gib():
    """Rows whose byte offsets pass 32 bits."""
    from paper_2307_02486_amd import paged_attn
    note("[paged8] large pool")
    pages, page, H, D = 37000, 64, 16, 128   # 4.85 GB each of k and v
    kc = torch.zeros((pages, H, page, D), dtype=torch.uint8, device="cuda").view(F8)
    vc = torch.zeros((pages, H, page, D), dtype=torch.uint8, device="cuda").view(F8)
    ks, vs = (torch.full((pages, H, 4), 127, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
    rng = np.random.default_rng(3)
    for new in ([1], [70]):
        n = 200 + new[0]
        ids = pages - 1 - rng.permutation(4000)[: -(-n // page)]
        small = normal_pool(len(ids), H, page, D, 5), normal_pool(len(ids), H, page, D, 6)
        at = torch.from_numpy(ids).cuda()
        for (c, s), (x, y) in zip(((kc, ks), (vc, vs)), small):
            c.view(torch.uint8)[at], s.view(torch.uint8)[at] = x.view(torch.uint8), y.view(torch.uint8)
        q = workloads.make_random((new[0], H, D), BF, 1.0, 5, "cuda", 0)
        dev = [at[None].to(torch.int32).contiguous(), torch.tensor([n], dtype=torch.int32, device="cuda"),
               torch.tensor([0, new[0]], dtype=torch.int32, device="cuda")]
        out, lse = paged_attn(q, kc, vc, *dev, [(128, 1), (512, 3)], k_scale=ks, v_scale=vs)
        compare(out, lse, q, [elements(*x) for x in small], np.arange(len(ids))[None], [n], [0, new[0]], page,
                [(128, 1), (512, 3)], BF, "large pool")


def test_starts_that_do_not_ascend_stay_in_bounds():
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    note("[paged8] starts that do not ascend")
    T, B, H, page, width = 40, 60, 12, 16, 64
    pats = [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)]
    (kc, ks), (vc, vs) = normal_pool(8, H, page, 64, 1), normal_pool(8, H, page, 64, 2)
    q = workloads.make_random((T, H, 64), BF, 1.0, 21, "cuda", 2)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width) % 10 - 1
    lens = torch.full((B,), 300, dtype=torch.int32, device="cuda")
    need = paged_workspace_bytes(T, B, H, H, 64, 8, page, width, pats)
    for far in (4, T):
        start = torch.tensor([far * (b % 2) for b in range(B + 1)], dtype=torch.int32, device="cuda")
        guard = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros((T + 8, H, 64), dtype=BF, device="cuda"), torch.zeros((H + 1, T), device="cuda")
        paged_attn(q, kc, vc, table, lens, start, pats, out=out[:T], lse=lse[:H], workspace=guard[:need], k_scale=ks,
                   v_scale=vs)
        torch.cuda.synchronize()
        assert bool((guard[need:] == 0x5A).all()) and bool((out[T:] == 0).all()) and bool((lse[H:] == 0).all())
