"""The attention that pages get from new tokens, against float64 on the values that
the cache holds.

Bars: a pair's weight is exp of a difference of float32 numbers of size |s| and
|lse| below 40 (in log2 units, a rounding of each, of their product with the scale
and of the exponential), so within 40 * 3 * 2^-24 * ln 2 + 2^-22 < 6e-6 of itself,
and so are sums of weights up to their own roundings: 2e-5 of a page's weight and
1e-6 more.  The lse are the reference's own, rounded to float32 (40 * 2^-24 ln 2
more, counted above)."""
import numpy as np
import pytest
import torch

import workloads
from oracle.compressed_ref import attention_ref, key_weights_ref
from tests.cache8 import E8, F8, normal_pool, rows_of
from tests.gpu_util import note, require_gpu, to64
from tests.test_paged8_gpu import DENSE, PAPER, held_values, setup

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


CASES = [
    # (new tokens, cached before, H, Hkv, D, page, patterns, dtype)
    ([1], [0], 1, 1, 64, 16, DENSE, BF),
    ([1], [2500], 12, 12, 64, 64, PAPER, BF),
    ([1, 1, 1], [0, 31, 700], 12, 12, 64, 16, [(64, 1), (256, 3), (1024, 5)], BF),
    ([1, 1], [1500, 600], 8, 2, 128, 32, DENSE, BF),
    ([1, 0, 1], [300, 5, 77], 24, 1, 64, 8, [(128, 1), (512, 2)], BF),     # more columns than a step of 16
    ([2, 0, 0], [20, 5, 7], 6, 3, 32, 16, [(128, 1), (300, 7)], BF),       # as many tokens as sequences, two of one
    ([1, 4, 2], [300, 5, 77], 24, 1, 64, 8, [(128, 1), (512, 2)], BF),
    ([3, 3], [100, 500], 6, 3, 32, 1, [(100, 1), (333, 7)], BF),           # pages of one token
    ([1, 2], [63, 64], 8, 4, 64, 64, [(64, 2), (128, 3), (512, 9)], BF),
    ([130], [0], 3, 3, 64, 16, [(64, 1), (128, 2)], BF),                   # several segments
    ([157], [600], 4, 2, 64, 64, [(300, 1), (700, 3), (1 << 30, 11)], BF),
    ([40], [2300], 2, 1, 128, 128, DENSE, BF),                             # more keys than are looked up at once
    ([60], [1200], 2, 2, 32, 1024, [(1 << 20, 1), (999, 5)], BF),          # few pages, of over a thousand tokens
    ([5], [2200], 1, 1, 32, 1, DENSE, BF),                                 # more pages than an item has
    ([64, 1, 90, 0, 3], [10, 900, 0, 50, 129], 12, 4, 64, 16, [(256, 1), (512, 2), (4096, 4)], BF),
    ([1] * 20 + [40] + [1] * 50, list(range(0, 710, 10)), 4, 4, 64, 32, [(128, 1), (512, 4)], BF),
    ([5, 4, 6, 1], [90, 80, 0, 7], 16, 4, 128, 16, [(64, 1), (4096, 2)], BF),
    ([1, 7, 40], [0, 300, 33], 6, 2, 32, 16, [(512, 1), (600, 3)], F32),
    ([1], [700], 4, 4, 64, 64, DENSE, F32),
    ([1, 33], [300, 0], 4, 1, 128, 8, [(64, 2), (128, 3)], F32),
    ([40, 2], [40, 3], 3, 3, 64, 16, [(16, 1), (48, 1), (1 << 20, 2)] + [(8 * i, i) for i in range(2, 15)], BF),
    ([1], [500], 3, 3, 64, 16, [(600, 40), (1 << 40, 1 << 33), (7, 1)], BF),
]


def reference(q, pools, table, lens, start, page, patterns, scale=None):
    """(lse [T, H], what each page of the pool gets [pages])."""
    q64, pages = to64(q), pools[0].shape[0]
    lse, got = np.full(q64.shape[:2], -np.inf), np.zeros(pages)
    for b, n in enumerate(lens):
        rows, new = slice(start[b], start[b + 1]), int(start[b + 1] - start[b])
        if new == 0:
            continue
        k, there = rows_of(pools[0], table[b], page, int(n))
        v, _ = rows_of(pools[1], table[b], page, int(n))
        lse[rows] = attention_ref(q64[rows], k, v, n - new, patterns, there, scale)[1]
        w = key_weights_ref(q64[rows], k, n - new, patterns, there, lse[rows], scale)
        at = np.flatnonzero(there)
        np.add.at(got, table[b][at // page], w[at])
    return lse, got


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:60])
@pytest.mark.parametrize("gone", [0.0, 0.3, 1.0], ids=str)
def test_matches_the_definition(case, gone):
    from paper_2307_02486_amd import page_weights
    new, before, H, Hkv, D, page, patterns, dtype = case
    note(f"[weights] {gone} {str(case)[:200]}")
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, before, H, Hkv, D, page, dtype, gone)
    lse64, want = reference(q, held_values(kc, vc, ks, vs), table, lens, start, page, patterns)
    lse = torch.from_numpy(lse64.T.astype(np.float32)).contiguous().cuda()
    had = torch.rand(kc.shape[0], device="cuda")
    weights = had.clone()
    assert page_weights(q, lse, kc, ks, *dev, patterns, weights) is weights
    torch.cuda.synchronize()
    got, old = to64(weights), to64(had)
    assert (np.abs(got - old - want) <= 2e-5 * want + 1e-6 + 2.0 ** -24 * got).all(), np.abs(got - old - want).max()
    assert np.array_equal(got[want == 0], old[want == 0])  # others are as they were
    again = had.clone()
    page_weights(q, lse, kc, ks, *dev, patterns, again)
    assert torch.equal(again, weights)


def test_each_row_gives_one():
    """With the attention's own lse; rows without keys give nothing."""
    from paper_2307_02486_amd import page_weights, paged_attn
    note("[weights] sums")
    for new in ([1, 1, 1], [200, 1, 30]):
        pats = [(128, 1), (512, 3), (2048, 12)]
        q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [900, 60, 10], 12, 4, 64, 16, BF)
        out, lse = paged_attn(q, kc, vc, *dev, pats, k_scale=ks, v_scale=vs)
        weights = torch.zeros(kc.shape[0], device="cuda")
        page_weights(q, lse, kc, ks, *dev, pats, weights)
        rows = int(torch.isfinite(lse).sum())
        assert abs(float(weights.double().sum()) - rows) <= 2e-5 * rows


def test_rows_with_an_lse_that_is_not_finite_give_nothing():
    from paper_2307_02486_amd import page_weights, paged_attn
    note("[weights] not finite")
    for new in ([1, 1], [40, 3]):
        q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [90, 50], 4, 4, 64, 16, BF, 0.0)
        kc.view(torch.uint8)[int(table[0, 1]), 2, 5, 7] = 0x7F  # a NaN that head 2 of the first sequence sees
        q[-1, 1, 0] = float("inf")
        out, lse = paged_attn(q, kc, vc, *dev, DENSE, k_scale=ks, v_scale=vs)
        bad = ~torch.isfinite(lse)
        assert int(bad.sum()) == new[0] + 1
        weights = torch.zeros(kc.shape[0], device="cuda")
        page_weights(q, lse, kc, ks, *dev, DENSE, weights)
        rows = 4 * sum(new) - new[0] - 1
        assert bool(torch.isfinite(weights).all()) and abs(float(weights.double().sum()) - rows) <= 2e-5 * rows


@pytest.mark.parametrize("new", [[1], [2, 90]], ids=str)
def test_strided_queries_scale_and_workspace(new):
    from paper_2307_02486_amd import page_weights, page_weights_workspace_bytes
    note(f"[weights] strided {new}")
    pats, H = [(64, 1), (256, 2)], 6
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, [70, 5][: len(new)], H, 2, 64, 16, BF)
    lse64, want = reference(q, held_values(kc, vc, ks, vs), table, lens, start, 16, pats, 0.3)
    lse = torch.from_numpy(lse64.T.astype(np.float32)).contiguous().cuda()
    wide = torch.full((q.shape[0], H + 5, 64), float("nan"), dtype=BF, device="cuda")
    wide[:, :H] = q
    need = page_weights_workspace_bytes(q.shape[0], len(new), H, 2, 64, kc.shape[0], 16, dev[0].shape[1], pats)
    guard = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    weights = torch.zeros(kc.shape[0], device="cuda")
    page_weights(wide[:, :H], lse, kc, ks, *dev, pats, weights, scale=0.3, workspace=guard[:need])
    torch.cuda.synchronize()
    assert bool((guard[need:] == 0x5A).all())
    assert (np.abs(to64(weights) - want) <= 2e-5 * want + 1e-6).all()


def test_nothing_new_and_tokens_of_no_sequence():
    from paper_2307_02486_amd import page_weights
    note("[weights] no place")
    q, kc, vc, ks, vs, dev, table, lens, start = setup([2, 3], [20, 9], 4, 4, 64, 16, BF, 0.0)
    weights = torch.ones(kc.shape[0], device="cuda")
    lse = torch.zeros((4, 5), device="cuda")
    page_weights(q[:0], lse[:, :0].contiguous(), kc, ks, dev[0], dev[1], torch.zeros_like(dev[2]), DENSE, weights)
    page_weights(q, lse, kc, ks, dev[0], torch.zeros_like(dev[1]), dev[2], DENSE, weights)
    page_weights(q, lse, kc, ks, dev[0], dev[1], torch.zeros_like(dev[2]), DENSE, weights)
    assert bool((weights == 1).all())


def test_starts_that_do_not_ascend_stay_in_bounds():
    from paper_2307_02486_amd import page_weights, page_weights_workspace_bytes
    note("[weights] starts that do not ascend")
    H, page, width, B = 12, 16, 64, 60
    pats = [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)]
    kc, ks = normal_pool(8, H, page, 64, 1)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width) % 10 - 1
    lens = torch.full((B,), 300, dtype=torch.int32, device="cuda")
    for T in (40, 90):
        q = workloads.make_random((T, H, 64), BF, 1.0, 21, "cuda", 2)
        lse = torch.zeros((H, T), device="cuda")
        need = page_weights_workspace_bytes(T, B, H, H, 64, 8, page, width, pats)
        for far in (4, T):
            start = torch.tensor([far * (b % 2) for b in range(B + 1)], dtype=torch.int32, device="cuda")
            guard = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
            weights = torch.zeros(16, device="cuda")
            page_weights(q, lse, kc, ks, table, lens, start, pats, weights[:8], workspace=guard[:need])
            torch.cuda.synchronize()
            assert bool((guard[need:] == 0x5A).all()) and bool((weights[8:] == 0).all())


def test_other_stream_and_graph_replays():
    """A captured step of attention and weights replayed with other lengths and
    tables, with eager work between: the same bits."""
    from paper_2307_02486_amd import page_weights, paged_attn
    note("[weights] graph")
    pats = [(64, 1), (256, 2)]
    for news in ([[1, 1, 1], [1, 1, 1], [0, 2, 1]], [[60, 2, 0], [1, 1, 60], [20, 22, 20]]):
        sets = [setup(n, [30 + 40 * i, 5, 90], 6, 3, 64, 16, BF, seed=i) for i, n in enumerate(news)]
        T, width, pages = sum(news[0]), max(s[5][0].shape[1] for s in sets), max(s[1].shape[0] for s in sets)
        table = torch.zeros((3, width), dtype=torch.int32, device="cuda")
        lens, start = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        q = torch.zeros((T, 6, 64), dtype=BF, device="cuda")
        pools = [torch.zeros((pages, 3, 16, 64), dtype=torch.uint8, device="cuda").view(F8) for _ in range(2)]
        scales = [torch.full((pages, 3, 1), 127, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2)]
        weights = torch.zeros(pages, device="cuda")

        def load(s):
            table.fill_(-1)
            table[:, : s[5][0].shape[1]] = s[5][0]
            lens.copy_(s[5][1]), start.copy_(s[5][2]), q.copy_(s[0])
            for x, y in zip(pools + scales, (s[1], s[2], s[3], s[4])):
                x.view(torch.uint8)[: y.shape[0]] = y.view(torch.uint8)
            weights.zero_()

        def call():
            out, lse = paged_attn(q, *pools, table, lens, start, pats, k_scale=scales[0], v_scale=scales[1])
            page_weights(q, lse, pools[0], scales[0], table, lens, start, pats, weights)
            return out, lse

        side = torch.cuda.Stream()
        load(sets[0])
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        warm = weights.clone()
        load(sets[0])
        call()
        assert torch.equal(warm, weights)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = call()
        for i in (0, 1, 2, 1, 0):
            load(sets[i])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (*held, weights)]
            load(sets[i])
            want = [*call(), weights]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_columns_dealt_out():
    """So many tokens and heads of a key head that several workgroups share them."""
    from paper_2307_02486_amd import page_weights
    note("[weights] columns dealt out")
    for new, before, H, Hkv, D, pats in (([700, 3], [100, 900], 8, 1, 64, [(1024, 1), (2048, 3)]),
                                         ([1500], [40], 4, 4, 32, DENSE)):
        q, kc, vc, ks, vs, dev, table, lens, start = setup(new, before, H, Hkv, D, 16, BF)
        lse64, want = reference(q, held_values(kc, vc, ks, vs), table, lens, start, 16, pats)
        lse = torch.from_numpy(lse64.T.astype(np.float32)).contiguous().cuda()
        weights = torch.zeros(kc.shape[0], device="cuda")
        page_weights(q, lse, kc, ks, *dev, pats, weights)
        assert (np.abs(to64(weights) - want) <= 2e-5 * want + 1e-6).all()


def test_pool_beyond_4_gib():
    """Rows whose byte offsets pass 32 bits: the weights that the same call gives in a small pool."""
    from paper_2307_02486_amd import page_weights
    note("[weights] large pool")
    pages, page, H, D = 37000, 64, 16, 128   # 4.85 GB
    large = torch.zeros((pages, H, page, D), dtype=torch.uint8, device="cuda").view(F8)
    scales = torch.full((pages, H, 4), 127, dtype=torch.uint8, device="cuda").view(E8)
    ids = torch.tensor([36999, 35001, 36000, 34000, 33001], dtype=torch.int32, device="cuda")
    small, small_scales = normal_pool(5, H, page, D, 5)
    large.view(torch.uint8)[ids.long()] = small.view(torch.uint8)
    scales.view(torch.uint8)[ids.long()] = small_scales.view(torch.uint8)
    for new in (1, 90):
        q = workloads.make_random((new, H, D), BF, 1.0, 5, "cuda", 0)
        lse = torch.full((H, new), 6.0, device="cuda")
        lens, start = (torch.tensor(i, dtype=torch.int32, device="cuda") for i in ([300], [0, new]))
        got, want = torch.zeros(pages, device="cuda"), torch.zeros(5, device="cuda")
        page_weights(q, lse, large, scales, ids[None].contiguous(), lens, start, [(128, 1), (512, 3)], got)
        page_weights(q, lse, small, small_scales, torch.arange(5, dtype=torch.int32, device="cuda")[None], lens, start,
                     [(128, 1), (512, 3)], want)
        assert bool((want > 0).any()) and torch.equal(got[ids.long()], want) and int((got != 0).sum()) == int((want != 0).sum())


def test_any_hint_of_the_most_new_tokens():
    """As many tokens as sequences or fewer, in one of them, some or all."""
    from paper_2307_02486_amd import page_weights
    note("[weights] hints")
    for new in ([40] + [0] * 59, [1, 3, 0, 0, 1], [1, 1, 1]):
        before = [500 + 7 * i for i in range(len(new))]
        for H, Hkv, pats in ((4, 4, [(128, 1), (512, 4)]), (8, 2, [(64, 1), (4096, 2)])):
            q, kc, vc, ks, vs, dev, table, lens, start = setup(new, before, H, Hkv, 64, 16, BF)
            lse64, want = reference(q, held_values(kc, vc, ks, vs), table, lens, start, 16, pats)
            lse = torch.from_numpy(lse64.T.astype(np.float32)).contiguous().cuda()
            for hint in (None, 1, 3, max(new), 1000):
                weights = torch.zeros(kc.shape[0], device="cuda")
                page_weights(q, lse, kc, ks, *dev, pats, weights, max_new=hint)
                assert (np.abs(to64(weights) - want) <= 2e-5 * want + 1e-6).all(), hint
