"""The append into a cache in 8 bits against the definition.

Without norm and rotation the inputs are the values themselves: every byte and
every scale is that of the reference.  With them the value before its rounding is
off by float32 arithmetic (angles reduced in float64; within 2e-6 of the row's
largest element): next to a tie it is rounded to e4m3's other neighbour, an eighth
of the leading power of two away, and next to 448 times a power of two the block
takes the other scale, at which every value still is within half a step (2^-4) of
it.  So every element is within 2^-3 of its size (or a step of the least normal
value, 2^-9 of the scale), and less than one in 200 differs at all: ties are as
far apart as steps, 2^-4 of a value at least, and 2e-6 of four times a value
around each is 2e-4 of them."""
import numpy as np
import pytest
import torch

import workloads
from oracle.paged_ref import heads_ref
from tests.cache8 import E8, F8, append_ref, bytes_of, elements, pool, unscaled
from tests.gpu_util import note, require_gpu, to64
from tests.test_heads_gpu import paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


CASES = [
    # (new tokens, cached before, H, Hkv, D, page, dtype)
    ([1], [0], 1, 1, 64, 16, BF),
    ([1, 1, 1, 1], [0, 15, 16, 40], 12, 12, 64, 64, BF),
    ([3, 40, 0, 1], [14, 5, 9, 31], 6, 2, 32, 8, BF),       # pages of fewer tokens than a block
    ([17, 2], [15, 30], 16, 4, 128, 32, BF),
    ([33], [7], 5, 5, 64, 1, BF),                           # pages of one token
    ([100, 1], [0, 3], 24, 24, 64, 16, BF),                 # more heads than a workgroup has at once
    ([1] * 70, list(range(70)), 4, 2, 64, 16, BF),          # over 64 sequences
    ([5, 20], [3, 12], 4, 2, 64, 16, F32),
    ([40, 3], [9, 0], 3, 1, 128, 256, F32),
    ([9, 30], [2, 1], 2, 2, 32, 2, F32),
]


def inputs(case, norm, sliced, sigma=1.0):
    new, before, H, Hkv, D, page, dtype = case
    table, lens, start, dev, pages = paged(new, before, page)
    x = workloads.make_random((int(start[-1]), H + 2 * Hkv, D), dtype, sigma, 61, "cuda", 0)
    q, k, v = x[:, :H], x[:, H: H + Hkv], x[:, H + Hkv:]
    if not sliced:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    w = [workloads.make_random((D,), dtype, 0.2, 62, "cuda", t) + 1 for t in (0, 1)] if norm else [None, None]
    (kc, ks), (vc, vs) = pool(pages, Hkv, page, D, 1), pool(pages, Hkv, page, D, 2)
    return table, lens, start, dev, q, k, v, w, kc, vc, ks, vs


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:50])
@pytest.mark.parametrize("sigma", [1.0, 100.0, 1e-3, 1e-30], ids=str)
def test_values_as_they_are(case, sigma):
    """Bit by bit; blocks with older tokens at scales below and above the new ones'."""
    from paper_2307_02486_amd import cache_append
    note(f"[append8] {case} {sigma}")
    table, lens, start, dev, q, k, v, _, kc, vc, ks, vs = inputs(case, False, sigma == 1.0, sigma)
    page = case[5]
    want = []
    for vals, scale, new in ((kc, ks, k), (vc, vs, v)):
        w, e = unscaled(vals), bytes_of(scale).astype(np.int64) - 127
        append_ref(w, e, table, lens, start, to64(new), page)
        want.append((w, e))
    out = cache_append(q, k, v, kc, vc, *dev, rotate=False, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert torch.equal(out, q)
    for vals, scale, (w, e) in ((kc, ks, want[0]), (vc, vs, want[1])):
        assert np.array_equal(bytes_of(scale).astype(np.int64) - 127, e)
        assert np.array_equal(unscaled(vals), w)


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:50])
@pytest.mark.parametrize("norm", [False, True], ids=str)
def test_keys_normed_and_rotated(case, norm):
    from paper_2307_02486_amd import cache_append
    note(f"[append8] rotated {case} {norm}")
    new, before, H, Hkv, D, page, dtype = case
    table, lens, start, dev, q, k, v, w, kc, vc, ks, vs = inputs(case, norm, norm)
    center = 20
    pos = np.concatenate([np.arange(c, c + n) for n, c in zip(new, before)])
    w64 = [None if x is None else to64(x) for x in w]
    k64 = heads_ref(to64(k), w64[1], pos, -1, center)
    wk, ek = unscaled(kc), bytes_of(ks).astype(np.int64) - 127
    append_ref(wk, ek, table, lens, start, k64, page)
    wv, ev = unscaled(vc), bytes_of(vs).astype(np.int64) - 127
    append_ref(wv, ev, table, lens, start, to64(v), page)
    out = cache_append(q, k, v, kc, vc, *dev, q_weight=w[0], k_weight=w[1], center=center, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    q64 = heads_ref(to64(q), w64[0], pos, 1, center)
    bar = (2.0 ** -8 * np.abs(q64) if dtype == BF else 0) + 4e-6 * np.abs(q64).max(-1, keepdims=True)
    assert (np.abs(to64(out) - q64) <= bar).all()
    assert np.array_equal(bytes_of(vs).astype(np.int64) - 127, ev) and np.array_equal(unscaled(vc), wv)
    size = page // ek.shape[2]
    scale = np.exp2(np.repeat(ek, size, axis=2))[..., None]
    ref, got = wk * scale, elements(kc, ks)
    off = np.abs(got - ref)
    assert (off <= 2.0 ** -3 * np.maximum(np.abs(ref), 2.0 ** -6 * scale)).all()
    assert (off > 0).sum() <= max(2, ref.size // 200)


def test_infinities_nan_and_extremes():
    """They become NaN where they are and leave their block's scale to the others."""
    from paper_2307_02486_amd import cache_append
    note("[append8] infinities")
    case = ([20, 3], [3, 0], 2, 2, 64, 16, F32)
    table, lens, start, dev, q, k, v, _, kc, vc, ks, vs = inputs(case, False, False)
    k[2, 0, 5], k[7, 1, 9], k[21, 0, 0] = float("inf"), float("nan"), float("-inf")
    v[0], v[1, 0], v[22] = 0.0, 1e38, 1e-42
    k[13, 1, 3] = -1.6e38
    want = []
    for vals, scale, new in ((kc, ks, k), (vc, vs, v)):
        w, e = unscaled(vals), bytes_of(scale).astype(np.int64) - 127
        append_ref(w, e, table, lens, start, to64(new), 16)
        want.append((w, e))
    cache_append(None, k, v, kc, vc, *dev, rotate=False, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    for vals, scale, (w, e) in ((kc, ks, want[0]), (vc, vs, want[1])):
        assert np.array_equal(bytes_of(scale).astype(np.int64) - 127, e)
        assert np.array_equal(unscaled(vals), w, equal_nan=True)
    assert np.isnan(unscaled(kc)).sum() == 3


def test_token_by_token_and_at_once():
    """Scales are the largest of a block's tokens either way; values that came before
    the largest are rounded a second time only where the scale then cuts them short."""
    from paper_2307_02486_amd import cache_append
    note("[append8] token by token")
    n, Hkv, D, page = 50, 3, 64, 32
    table, lens, start, dev, pages = paged([n], [0], page)
    k, v = (workloads.make_random((n, Hkv, D), BF, 1.0, 63, "cuda", t) for t in (0, 1))
    k *= torch.exp2(torch.arange(n, device="cuda") % 7).to(BF)[:, None, None]
    pools = []
    for steps in ([n], [1] * n, [13, 1, 20, 16]):
        kc, vc = (torch.zeros((pages, Hkv, page, D), device="cuda").to(F8) for _ in range(2))
        ks, vs = (torch.full((pages, Hkv, 2), 200, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
        at = 0
        for m in steps:
            at += m
            cache_append(None, k[at - m: at], v[at - m: at], kc, vc, dev[0],
                         torch.tensor([at], dtype=torch.int32, device="cuda"),
                         torch.tensor([0, m], dtype=torch.int32, device="cuda"), rotate=False, k_scale=ks, v_scale=vs)
        torch.cuda.synchronize()
        pools.append((elements(kc, ks), elements(vc, vs), bytes_of(ks), bytes_of(vs)))
    for other in pools[1:]:
        for a, b, s in ((pools[0][0], other[0], other[2]), (pools[0][1], other[1], other[3])):
            unit = np.exp2(np.repeat(s.astype(np.float64) - 127, 16, axis=2))[..., None]
            assert (np.abs(a - b) <= 2.0 ** -9 * unit).all()  # a step below e4m3's least normal value
        assert np.array_equal(pools[0][2], other[2]) and np.array_equal(pools[0][3], other[3])


def test_rows_and_pages_without_a_place():
    """Tokens of no sequence have zero queries and are not cached; pages outside the
    pool are not written; all else stays as it was."""
    from paper_2307_02486_amd import cache_append
    note("[append8] no place")
    case = ([3, 4], [20, 9], 4, 2, 64, 16, BF)
    table, lens, start, dev, q, k, v, _, kc, vc, ks, vs = inputs(case, False, False)
    more = [torch.cat([x, x]) for x in (q, k, v)]
    before = [bytes_of(x).copy() for x in (kc, vc, ks, vs)]
    bad = dev[0].clone()
    bad[0] = -1
    bad[1] = kc.shape[0]
    out = cache_append(*more, kc, vc, bad, *dev[1:], center=8, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, bytes_of(x)) for a, x in zip(before, (kc, vc, ks, vs)))
    assert bool((out[7:] == 0).all()) and bool((out[:7] != 0).any(-1).all())
    short, far = dev[1].clone(), dev[1].clone()
    short[0], far[1] = 1, dev[0].shape[1] * 16 + 2  # tokens before position 0, past the table
    table2 = dev[0].clamp(max=kc.shape[0] - 1)
    for L, gone in ((short, [0, 1]), (far, [5, 6])):
        out = cache_append(q, k, v, kc, vc, table2, L, dev[2], center=8, k_scale=ks, v_scale=vs)
        torch.cuda.synchronize()
        assert bool((out[gone] == 0).all())
    cache_append(q, k, v, kc, vc, table2, dev[1], dev[2].flip(0).contiguous(), center=8, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()


def test_other_stream_and_graph_replays():
    """A captured append replayed with other lengths, tables and tokens, with eager
    work between: the bytes of the eager one."""
    from paper_2307_02486_amd import cache_append
    note("[append8] graph")
    H, Hkv, D, page, T = 4, 2, 64, 16, 30
    sets = []
    for i, (new, before) in enumerate((([28, 2], [3, 40]), ([1, 29], [15, 0]), ([15, 15], [1, 17]))):
        table, lens, start, dev, pages = paged(new, before, page, seed=i)
        sets.append((dev, pages))
    pages, width = max(s[1] for s in sets), max(s[0][0].shape[1] for s in sets)
    table = torch.zeros((2, width), dtype=torch.int32, device="cuda")
    lens, start = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((T, h, D), dtype=BF, device="cuda") for h in (H, Hkv, Hkv))
    first = [*pool(pages, Hkv, page, D, 3), *pool(pages, Hkv, page, D, 4)]
    kc, ks, vc, vs = (torch.empty_like(x.view(torch.uint8)).view(x.dtype) for x in first)

    def load(i):
        dev = sets[i][0]
        table.zero_()
        table[:, : dev[0].shape[1]] = dev[0].clamp(max=pages - 1)
        lens.copy_(dev[1]), start.copy_(dev[2])
        for t, x in enumerate((q, k, v)):
            x.copy_(workloads.make_random(x.shape, BF, 1.0, 700 + i, "cuda", t))
        for x, f in zip((kc, ks, vc, vs), first):
            x.view(torch.uint8).copy_(f.view(torch.uint8))

    def call():
        return cache_append(q, k, v, kc, vc, table, lens, start, center=30, k_scale=ks, v_scale=vs)

    def all_bytes(out):
        return [out.clone()] + [x.view(torch.uint8).clone() for x in (kc, ks, vc, vs)]

    side = torch.cuda.Stream()
    load(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = call()
    torch.cuda.current_stream().wait_stream(side)
    warm = all_bytes(warm)
    load(0)
    assert all(torch.equal(a, b) for a, b in zip(warm, all_bytes(call())))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in (0, 1, 2, 1, 0):
        load(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = all_bytes(held)
        load(i)
        want = all_bytes(call())
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_pool_beyond_4_gib():
    """Rows whose byte offsets pass 32 bits: what the same call leaves in a small pool."""
    from paper_2307_02486_amd import cache_append
    note("[append8] large pool")
    pages, page, H, D = 37000, 64, 16, 128   # 4.85 GB each of k and v
    large = [torch.zeros((pages, H, page, D), dtype=torch.uint8, device="cuda").view(F8) for _ in range(2)]
    scales = [torch.zeros((pages, H, 4), dtype=torch.uint8, device="cuda").view(E8) for _ in range(2)]
    ids = torch.tensor([36999, 35001, 36000], dtype=torch.int32, device="cuda")
    small = [torch.zeros((3, H, page, D), dtype=torch.uint8, device="cuda").view(F8) for _ in range(2)]
    small_scales = [torch.zeros((3, H, 4), dtype=torch.uint8, device="cuda").view(E8) for _ in range(2)]
    for n0, n1 in ((0, 150), (150, 151)):
        x = workloads.make_random((n1 - n0, 2 * H, D), BF, 1.0, 9, "cuda", n0)
        lens, start = (torch.tensor(i, dtype=torch.int32, device="cuda") for i in ([n1], [0, n1 - n0]))
        for pools, sc, table in ((large, scales, ids), (small, small_scales, torch.arange(3, dtype=torch.int32, device="cuda"))):
            cache_append(None, x[:, :H], x[:, H:], *pools, table[None].contiguous(), lens, start,
                         k_scale=sc[0], v_scale=sc[1])
    for a, b in zip(large + scales, small + small_scales):
        a, b = a.view(torch.uint8), b.view(torch.uint8)
        assert bool((b != 0).any()) and torch.equal(a[ids.long()], b)
        assert int(torch.count_nonzero(a)) == int(torch.count_nonzero(b))
