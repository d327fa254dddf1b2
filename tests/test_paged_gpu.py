"""Dilated attention over a paged cache against float64, every row.

Bars: bf16, |out - ref| <= 5e-3 max|v| (probabilities and out rounded to bf16,
2^-8 each at most and half that on average, rows kept as fp16 within 2^-11 of
their largest element, float32 sums; out is well below max|v| where many keys
share it) and |lse - ref| <= 1e-4 (float32 sums of D products of size
|q k|: for q, k ~ N(0, 1) below 1e-5, and the same for the sum of a few thousand
exponentials); float32, 2e-5 max|v| and 1e-4 (the products' roundings alone)."""
import numpy as np
import pytest
import torch

import workloads
from oracle.paged_ref import paged_attention_ref
from tests.gpu_util import note, require_gpu, to64
from tests.test_heads_gpu import paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
PAPER = [(2048, 1), (4096, 2), (8192, 4), (16384, 6), (32768, 12)]
DENSE = [(1 << 20, 1)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def setup(new, before, H, Hkv, D, page, dtype, seed=0, sigma=1.0):
    """Sequences with pages in random order; the pool is NaN wherever no sequence has a token."""
    table, lens, start, dev, pages = paged(new, before, page, seed=seed)
    T = int(start[-1])
    q = workloads.make_random((max(T, 1), H, D), dtype, sigma, 300 + seed, "cuda", 0)[:T]
    kc = torch.full((pages, Hkv, page, D), float("nan"), dtype=dtype, device="cuda")
    vc = kc.clone()
    seqs = []
    for b, length in enumerate(lens):
        k, v = (workloads.make_random((max(int(length), 1), Hkv, D), dtype, sigma if t == 1 else 1.0, 400 + seed + 7 * b,
                                      "cuda", t)[:length] for t in (1, 2))
        at = torch.arange(int(length), device="cuda")
        p = torch.from_numpy(table[b].astype(np.int64)).cuda()[at // page]
        kc[p, :, at % page], vc[p, :, at % page] = k, v
        seqs.append((k, v))
    return q, kc, vc, dev, lens, start, seqs


def compare(out, lse, q, seqs, lens, start, patterns, dtype, tag, scale=None):
    to, tl = (5e-3, 1e-4) if dtype == BF else (2e-5, 1e-4)
    out, lse, q64 = to64(out), to64(lse).T, to64(q)
    for b, (k, v) in enumerate(seqs):
        rows = slice(start[b], start[b + 1])
        n = start[b + 1] - start[b]
        if n == 0:
            continue
        v64 = to64(v)
        ro, rl = paged_attention_ref(q64[rows], to64(k), v64, lens[b] - n, patterns, scale)
        assert np.array_equal(np.isneginf(rl), np.isneginf(lse[rows])), f"{tag} {b}: rows without keys"
        assert not np.isnan(out[rows]).any() and not np.isnan(lse[rows]).any(), f"{tag} {b}: NaN"
        assert (out[rows][np.isneginf(rl)] == 0).all(), f"{tag} {b}: rows without keys are zero"
        eo = np.abs(out[rows] - ro).max() / max(np.abs(v64).max(), 1e-30)
        fin = np.isfinite(rl)
        el = np.abs(lse[rows][fin] - rl[fin]).max() if fin.any() else 0.0
        assert eo <= to and el <= tl, f"{tag} {b}: out {eo:.2e} (bar {to}), lse {el:.2e} (bar {tl})"


CASES = [
    # (new tokens, cached before, H, Hkv, D, page, patterns, dtype)
    ([1], [0], 1, 1, 64, 16, DENSE, BF),                                     # the first token
    ([1], [4095], 12, 12, 64, 64, PAPER, BF),
    ([1, 1, 1], [0, 31, 700], 12, 12, 64, 16, [(64, 1), (256, 3), (1024, 5)], BF),
    ([1, 1], [1500, 2600], 8, 2, 128, 32, DENSE, BF),                        # shared key heads; over a thousand keys a split
    ([1, 4, 2], [300, 5, 77], 24, 1, 64, 8, [(128, 1), (512, 2)], BF),       # more query heads to a key head than a tile's rows
    ([3, 3], [100, 1000], 6, 3, 32, 1, [(100, 1), (333, 7)], BF),            # pages of one token
    ([1, 2], [63, 64], 8, 4, 64, 64, [(64, 2), (128, 3), (512, 9)], BF),     # no pattern keeps every row
    ([2, 1], [40, 90], 5, 5, 64, 16, [(32, 1), (32, 1), (96, 1), (64, 2)], BF),  # repeated and crossing patterns
    ([1], [500], 3, 3, 64, 16, [(600, 40), (1 << 40, 1 << 33), (7, 1)], BF),  # dilations beyond the heads and the table
    ([5], [0], 4, 4, 64, 16, DENSE, BF),                                     # a lone sequence of few: tiles
    ([130], [0], 3, 3, 64, 16, [(64, 1), (128, 2)], BF),
    ([257], [1000], 4, 2, 64, 64, [(300, 1), (700, 3), (1 << 30, 11)], BF),
    ([70], [4500], 2, 1, 128, 128, DENSE, BF),                               # more keys than are looked up at once
    ([300], [17], 6, 6, 32, 8, [(100, 2), (400, 5)], BF),                    # rows without keys in tiles
    ([64, 1, 200, 0, 3], [10, 2000, 0, 50, 129], 12, 4, 64, 16, [(256, 1), (512, 2), (4096, 4)], BF),
    ([1] * 20 + [90] + [1] * 50, list(range(0, 710, 10)), 4, 4, 64, 32, [(128, 1), (512, 4)], BF),  # over 64 sequences
    ([20] * 66, [5] * 66, 2, 2, 64, 16, [(16, 1), (64, 4)], BF),
    ([300] + [1] * 39, list(range(0, 400, 10)), 12, 12, 64, 16, [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)], BF),
    ([20] * 66, list(range(66)), 12, 12, 64, 16, [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)], BF),  # more items than workgroups
    ([5, 4, 6, 1], [90, 80, 0, 7], 16, 4, 128, 16, [(64, 1), (4096, 2)], BF),  # both sides of the few
    ([1, 7, 40], [0, 600, 33], 6, 2, 32, 16, [(512, 1), (600, 3)], F32),
    ([3], [1000], 4, 4, 64, 64, DENSE, F32),
    ([1, 33], [300, 0], 4, 1, 128, 8, [(64, 2), (128, 3)], F32),
    ([2], [40], 17, 17, 64, 16, [(16, 1), (48, 1), (1 << 20, 2)] + [(8 * i, i) for i in range(2, 15)], BF),  # 16 patterns
    ([40, 2], [40, 3], 3, 3, 64, 16, [(16, 1), (48, 1), (1 << 20, 2)] + [(8 * i, i) for i in range(2, 15)], BF),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:60])
def test_matches_the_definition(case):
    from paper_2307_02486_amd import paged_attn
    new, before, H, Hkv, D, page, patterns, dtype = case
    note(f"[paged] {str(case)[:200]}")
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, dtype)
    out, lse = paged_attn(q, kc, vc, *dev, patterns)
    hint = paged_attn(q, kc, vc, *dev, patterns, max_new=max(new))
    wrong = paged_attn(q, kc, vc, *dev, patterns, max_new=1)
    torch.cuda.synchronize()
    compare(out, lse, q, seqs, lens, start, patterns, dtype, "no hint")
    compare(*hint, q, seqs, lens, start, patterns, dtype, "hint")
    compare(*wrong, q, seqs, lens, start, patterns, dtype, "a hint of one whatever the lengths")
    again = paged_attn(q, kc, vc, *dev, patterns)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("D", [32, 64, 128])
def test_matches_the_whole_sequence_operator(D):
    """Rows of chunks and single tokens are those of dilated_attn on the sequence."""
    from paper_2307_02486_amd import dilated_attn, paged_attn
    note(f"[paged] whole sequence D={D}")
    N, H, pats = 1337, 6, [(256, 1), (1000, 3)]
    q, kc, vc, dev, lens, start, seqs = setup([N], [0], H, H, D, 32, BF)
    want, want_lse = dilated_attn(q[None], seqs[0][0][None].contiguous(), seqs[0][1][None].contiguous(), pats)
    for lo, hi in ((0, N), (0, 1), (N - 1, N), (200, 203), (500, 900)):
        d = [dev[0], torch.tensor([hi], dtype=torch.int32, device="cuda"),
             torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda")]
        out, lse = paged_attn(q[lo:hi], kc, vc, *d, pats)
        scale = float(seqs[0][1].abs().max())
        assert float((out - want[0, lo:hi]).abs().max()) <= 1e-2 * scale
        assert float((lse - want_lse[0, :, lo:hi]).abs().max()) <= 2e-4


@pytest.mark.parametrize("new", [[1], [2, 90]], ids=str)
def test_strided_queries_given_outputs_and_scale(new):
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    note(f"[paged] strided {new}")
    pats, H = [(64, 1), (256, 2)], 6
    q, kc, vc, dev, lens, start, seqs = setup(new, [70, 5][: len(new)], H, 2, 64, 16, BF)
    T = q.shape[0]
    wide = torch.full((T, H + 5, 64), float("nan"), dtype=BF, device="cuda")
    wide[:, :H] = q
    out = torch.full((T, H, 64), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((H, T), float("nan"), device="cuda")
    need = paged_workspace_bytes(T, len(new), H, 2, 64, kc.shape[0], 16, dev[0].shape[1], pats)
    guard = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    got = paged_attn(wide[:, :H], kc, vc, *dev, pats, scale=0.3, out=out, lse=lse, workspace=guard[:need])
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse and bool((guard[need:] == 0x5A).all())
    compare(out, lse, q, seqs, lens, start, pats, BF, "strided", 0.3)


def test_tokens_of_no_sequence_and_lengths_that_do_not_fit():
    """Zeros and minus infinity for tokens past the last sequence and for those
    before position 0 or past the table, in both ways of computing."""
    from paper_2307_02486_amd import paged_attn
    note("[paged] no place")
    for new in ([2, 3], [30, 3], [30, 50]):
        q, kc, vc, dev, lens, start, seqs = setup(new, [20, 9], 4, 4, 64, 16, BF)
        T = sum(new)
        wide = workloads.make_random((T + 9, 4, 64), BF, 1.0, 77, "cuda", 0)
        wide[:T] = q
        short = dev[1].clone()
        short[0] = 1  # one token of the first sequence's has a position
        out, lse = paged_attn(wide, kc, vc, dev[0], short, dev[2], [(64, 1), (256, 2)])
        gone = list(range(new[0] - 1)) + list(range(T, T + 9))
        assert bool((out[gone] == 0).all()) and bool(torch.isneginf(lse[:, gone]).all())
        assert bool(torch.isfinite(out[new[0]: T].float()).all())
        far = dev[1].clone()
        far[1] = dev[0].shape[1] * 16 + 2  # the last two tokens lie past the table
        kc2, vc2 = torch.nan_to_num(kc), torch.nan_to_num(vc)
        table = dev[0].clamp(max=kc.shape[0] - 1)
        out, lse = paged_attn(wide[:T], kc2, vc2, table, far, dev[2], [(64, 1), (256, 2)])
        assert bool((out[T - 2:] == 0).all()) and bool(torch.isneginf(lse[:, T - 2:]).all())
        assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse[:, : T - 2]).all())


def test_pages_outside_the_pool_are_not_read():
    """Such entries read the pool's last page: finite results from a finite pool."""
    from paper_2307_02486_amd import paged_attn
    note("[paged] bad pages")
    for new in ([1, 1], [40, 1], [40, 60]):
        q, kc, vc, dev, *_ = setup(new, [50, 90], 4, 4, 64, 16, BF)
        table = dev[0].clone()
        table[:, ::2] = torch.tensor([-7, 1 << 30], dtype=torch.int32, device="cuda")[:, None]
        out, lse = paged_attn(q, torch.nan_to_num(kc), torch.nan_to_num(vc), table, *dev[1:], [(64, 1), (256, 2)])
        assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("new", [[1, 1], [100, 2]], ids=str)
def test_scores_that_grow_and_overflow(new):
    """Keys whose scores grow along the sequence far past every reference taken
    before, and keys whose scores overflow to minus infinity beside finite ones."""
    from paper_2307_02486_amd import paged_attn
    note(f"[paged] growing {new}")
    pats = [(1024, 1), (4096, 2)]
    q, kc, vc, dev, lens, start, seqs = setup(new, [700, 900], 4, 4, 64, 16, BF)
    q[:] = 0
    q[:, :, 0] = 1.0
    for b, (k, v) in enumerate(seqs):
        n = k.shape[0]
        at = torch.arange(n, device="cuda")
        ramp = (at.float() * 64).to(BF)  # scores of 8 a token: up to some thousands
        k[:] = 0
        k[:, :, 0] = ramp[:, None]
        p = dev[0][b].long()[at // 16]
        kc[p, :, at % 16] = k
    out, lse = paged_attn(q, kc, vc, *dev, pats)
    # scores of thousands in float32: lse within 2^-24 of them and out as before
    o64, l64 = to64(out), to64(lse).T
    for b, (k, v) in enumerate(seqs):
        rows = slice(start[b], start[b + 1])
        ro, rl = paged_attention_ref(to64(q[rows]), to64(k), to64(v), lens[b] - new[b], pats)
        assert np.abs(o64[rows] - ro).max() <= 5e-3 * np.abs(to64(v)).max()
        assert np.abs(l64[rows] - rl)[np.isfinite(rl)].max() <= 4e-3
    q[:, :, 1] = 1e20
    for b, (k, v) in enumerate(seqs):
        n = k.shape[0]
        at = torch.arange(n, device="cuda")
        k[:, :, 0] = (torch.sin(at.float()) * 8).to(BF)[:, None]
        k[:, :, 1] = torch.where(at % 3 == 1, -1e20, 0.0).to(BF)[:, None]
        k[: n // 2, :, 1] = -1e20  # the first half has no finite score
        k[n - 1, :, 1] = 0
        p = dev[0][b].long()[at // 16]
        kc[p, :, at % 16] = k
    out, lse = paged_attn(q, kc, vc, *dev, pats)
    o64, l64 = to64(out), to64(lse).T
    for b, (k, v) in enumerate(seqs):
        first = lens[b] - new[b]
        for i in range(new[b]):
            keep = to64(k)[:, 0, 1] == 0
            keep[first + i + 1:] = False
            k64, v64 = to64(k), to64(v)
            from oracle.paged_ref import counts
            c = counts(first + i, len(keep), 4, pats) * keep
            for h in range(4):
                sel = np.flatnonzero(c[h])
                if not sel.size:
                    continue
                s = k64[sel, h, 0] * 0.125
                w = c[h, sel] * np.exp(s - s.max())
                row = start[b] + i
                assert np.abs(o64[row, h] - w @ v64[sel, h] / w.sum()).max() <= 5e-3 * np.abs(v64).max()
                assert abs(l64[row, h] - (s.max() + np.log(w.sum()))) <= 1e-4


def test_large_value_rows():
    """Values of 1e5 and 1e-6, and rows far beyond fp16's range, keep bf16's precision."""
    from paper_2307_02486_amd import paged_attn
    note("[paged] value range")
    for new in ([1], [80]):
        q, kc, vc, dev, lens, start, seqs = setup(new, [300], 4, 4, 64, 16, BF)
        for factor in (1e5, 1e-6, 1e30):
            v = (seqs[0][1].float() * factor).to(BF)
            out, lse = paged_attn(q, kc, (vc.float() * factor).to(BF), *dev, [(128, 1), (512, 2)])
            compare(out, lse, q, [(seqs[0][0], v)], lens, start, [(128, 1), (512, 2)], BF, f"values {factor}")


def test_pool_beyond_4_gib():
    """Rows whose byte offsets pass 32 bits."""
    from paper_2307_02486_amd import paged_attn
    note("[paged] large pool")
    pages, page, H, D = 37000, 64, 16, 64   # 4.85 GB each of k and v
    kc = torch.zeros((pages, H, page, D), dtype=BF, device="cuda")
    vc = torch.zeros_like(kc)
    rng = np.random.default_rng(3)
    for new in ([1], [70]):
        n = 200 + new[0]
        ids = pages - 1 - rng.permutation(4000)[: -(-n // page)]
        table = torch.tensor(ids[None], dtype=torch.int32, device="cuda")
        k, v, q = (workloads.make_random((n, H, D), BF, 1.0, 5, "cuda", t) for t in range(3))
        at = torch.arange(n, device="cuda")
        kc[table[0].long()[at // page], :, at % page], vc[table[0].long()[at // page], :, at % page] = k, v
        lens, start = np.array([n]), np.array([0, new[0]])
        dev = [table, torch.tensor([n], dtype=torch.int32, device="cuda"),
               torch.tensor([0, new[0]], dtype=torch.int32, device="cuda")]
        out, lse = paged_attn(q[: new[0]], kc, vc, *dev, [(128, 1), (512, 3)])
        compare(out, lse, q[: new[0]], [(k, v)], lens, start, [(128, 1), (512, 3)], BF, "large pool")


def test_nothing_new():
    from paper_2307_02486_amd import paged_attn
    q, kc, vc, dev, *_ = setup([1], [3], 2, 2, 64, 16, BF)
    out, lse = paged_attn(q[:0], kc, vc, dev[0], dev[1], torch.zeros_like(dev[2]), DENSE)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)


def test_other_stream_and_graph_replays():
    """The same bits on another stream, and a captured call replayed with other
    lengths, tables and caches, with eager work between the replays."""
    from paper_2307_02486_amd import cache_append, paged_attn
    note("[paged] stream and graph")
    pats = [(64, 1), (256, 2)]
    for counts_ in ([[1, 1, 1], [1, 1, 1], [1, 1, 1]], [[60, 2, 0], [1, 1, 60], [20, 22, 20]]):
        sets = [setup(n, [30 + 40 * i, 5, 90], 6, 3, 64, 16, BF, seed=i) for i, n in enumerate(counts_)]
        T = sum(counts_[0])
        width = max(s[3][0].shape[1] for s in sets)
        pages = max(s[1].shape[0] for s in sets)
        table = torch.zeros((3, width), dtype=torch.int32, device="cuda")
        lens, start = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        kc = torch.zeros((pages, 3, 16, 64), dtype=BF, device="cuda")
        vc = torch.zeros_like(kc)
        q, kn, vn = (torch.zeros((T, h, 64), dtype=BF, device="cuda") for h in (6, 3, 3))

        def load(s, i):
            table.zero_()
            table[:, : s[3][0].shape[1]] = s[3][0].clamp(max=pages - 1)
            lens.copy_(s[3][1])
            start.copy_(s[3][2])
            kc.zero_(), vc.zero_()
            kc[: s[1].shape[0]].copy_(torch.nan_to_num(s[1]))
            vc[: s[2].shape[0]].copy_(torch.nan_to_num(s[2]))
            for t, x in enumerate((q, kn, vn)):
                x.copy_(workloads.make_random(x.shape, BF, 1.0, 500 + i, "cuda", t))

        def call():
            qo = cache_append(q, kn, vn, kc, vc, table, lens, start, center=64)
            return (qo, *paged_attn(qo, kc, vc, table, lens, start, pats, max_new=max(map(max, counts_))))

        load(sets[0], 0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            warm = call()
        torch.cuda.current_stream().wait_stream(side)
        load(sets[0], 0)
        here = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(warm, here))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = call()
        for i in (0, 1, 2, 1, 0):
            load(sets[i], i)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in held]
            load(sets[i], i)
            want = call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_starts_that_do_not_ascend_stay_in_bounds():
    """q_start names rows twice, more of them than there are tokens: nothing past
    the workspace and the outputs is written."""
    from paper_2307_02486_amd import paged_attn, paged_workspace_bytes
    note("[paged] starts that do not ascend")
    T, B, H, page, width = 40, 60, 12, 16, 64
    pats = [(64, 1), (128, 2), (256, 4), (512, 6), (512, 12)]
    kc, vc = (workloads.make_random((8, H, page, 64), BF, 1.0, 21, "cuda", t) for t in (0, 1))
    q = workloads.make_random((T, H, 64), BF, 1.0, 21, "cuda", 2)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width) % 8
    lens = torch.full((B,), 300, dtype=torch.int32, device="cuda")
    need = paged_workspace_bytes(T, B, H, H, 64, 8, page, width, pats)
    for far in (4, T):  # tokens by themselves, in tiles
        start = torch.tensor([far * (b % 2) for b in range(B + 1)], dtype=torch.int32, device="cuda")
        guard = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros((T + 8, H, 64), dtype=BF, device="cuda"), torch.zeros((H + 1, T), device="cuda")
        paged_attn(q, kc, vc, table, lens, start, pats, out=out[:T], lse=lse[:H], workspace=guard[:need])
        torch.cuda.synchronize()
        assert bool((guard[need:] == 0x5A).all()) and bool((out[T:] == 0).all()) and bool((lse[H:] == 0).all())


SPLIT = [
    # keys in several splits: (new tokens, cached before, H, Hkv, D, page, patterns)
    ([100], [1500], 3, 3, 64, 16, [(2048, 1), (2048, 2), (4096, 1), (1024, 1), (3000, 2), (5000, 3)]),  # few rows, six patterns
    ([900], [700], 12, 4, 64, 64, [(2048, 1), (2048, 2), (4096, 1), (1024, 1), (3000, 2), (5000, 3)]),  # many rows
    ([200], [1900], 6, 6, 32, 16, [(4096, 1), (1024, 3)]),
    ([60, 1, 1], [1200, 3000, 40], 4, 2, 128, 32, [(512, 1), (4096, 1)]),
    ([1, 1, 1], [5000, 300, 255], 6, 2, 64, 16, DENSE),
]


@pytest.mark.parametrize("case", SPLIT, ids=lambda c: str(c)[:60])
def test_split_keys(case):
    from paper_2307_02486_amd import paged_attn
    new, before, H, Hkv, D, page, patterns = case
    note(f"[paged] split {str(case)[:200]}")
    q, kc, vc, dev, lens, start, seqs = setup(new, before, H, Hkv, D, page, BF)
    for order in (patterns, patterns[::-1]):
        compare(*paged_attn(q, kc, vc, *dev, order, max_new=max(new)), q, seqs, lens, start, order, BF, "split")
