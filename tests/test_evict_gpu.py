"""Eviction against sorting: whole numbers, equal."""
import numpy as np
import pytest
import torch

from oracle.compressed_ref import evict_ref
from tests.gpu_util import note, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def check(weights, table, lens, page, keep, first, last):
    from paper_2307_02486_amd import evict_pages
    dev = [torch.from_numpy(x).cuda() for x in (weights, table, lens)]
    got = evict_pages(*dev, page, keep, first=first, last=last)
    torch.cuda.synchronize()
    want = evict_ref(weights, table, lens, page, keep, first, last)
    for name, g, w in zip(("table", "freed", "count"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert np.array_equal(dev[1].cpu().numpy(), table)
    return got


def case(B, most, page, seed, ties, gone=0.2):
    rng = np.random.default_rng(seed)
    pool = B * most + 5
    table = rng.permutation(pool)[: B * most].reshape(B, most).astype(np.int32)
    table[rng.random(table.shape) < gone] = -1
    table[rng.random(table.shape) < gone / 4] = 2 ** 30
    lens = rng.integers(0, most * page + 1, B).astype(np.int32)
    lens[0] = most * page
    w = np.exp(rng.normal(size=pool) * 8).astype(np.float32)
    if ties == "few":
        w = np.floor(w * 4).astype(np.float32) / 4
    elif ties == "all":
        w[:] = 0.5
    elif ties == "signs":
        with np.errstate(invalid="ignore"):
            w = (rng.integers(-3, 4, pool) * rng.choice([0.0, -0.0, 1.0, np.nan, np.inf], pool)).astype(np.float32)
    return w, table, lens


@pytest.mark.parametrize("B, most, page", [(1, 1, 16), (3, 7, 1), (5, 64, 64), (64, 100, 16), (2, 1024, 8), (2, 1025, 8),
                                           (1, 20000, 4)], ids=str)
@pytest.mark.parametrize("ties", ["none", "few", "all", "signs"], ids=str)
def test_matches_sorting(B, most, page, ties):
    note(f"[evict] {B} {most} {page} {ties}")
    w, table, lens = case(B, most, page, B + most, ties)
    for keep in sorted({0, 1, most // 3, most - 1, most + 5}):
        for first, last in ((0, 0), (1, 1), (4, 9), (most, 0), (0, most + 3)):
            check(w, table, lens, page, keep, first, last)


def test_weights_that_differ_in_one_digit():
    """Neighbours of one another in float32, so that every digit decides."""
    note("[evict] digits")
    rng = np.random.default_rng(1)
    for base in (0x00000001, 0x3F7FFFF0, 0x3F800000, 0x7F7FFF00):
        for shift in (0, 8, 16, 23):
            bits = (base + (rng.permutation(200).astype(np.int64) << shift)) & 0x7F7FFFFF
            w = bits.astype(np.uint32).view(np.float32)
            w[::3] *= -1
            table = rng.permutation(200).astype(np.int32)[None]
            check(w, table, np.array([200 * 4], np.int32), 4, 77, 0, 0)


def test_lengths_that_do_not_fit_the_table():
    note("[evict] lengths")
    w, table, lens = case(4, 30, 16, 3, "none")
    lens[:] = -5, 0, 30 * 16 + 999, 1
    check(w, table, lens, 16, 4, 1, 1)


def test_other_stream_and_graph_replays():
    from paper_2307_02486_amd import evict_pages
    note("[evict] graph")
    sets = [[torch.from_numpy(x).cuda() for x in case(6, 200, 16, i, "few")] for i in range(3)]
    w, table, lens = (torch.empty_like(x) for x in sets[0])

    def load(i):
        for x, y in zip((w, table, lens), sets[i]):
            x.copy_(y)

    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = evict_pages(w, table, lens, 16, 20)
    given = evict_pages(w, table, lens, 16, 20, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(warm, given))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = evict_pages(w, table, lens, 16, 20)
    for i in (0, 1, 2, 1, 0):
        load(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = evict_pages(w, table, lens, 16, 20)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_in_place_and_more_to_keep_than_there_can_be():
    from paper_2307_02486_amd import _lib, evict_pages
    note("[evict] in place")
    lib = _lib.load()
    for B, most in ((5, 70), (1, 20000)):
        w, table, lens = case(B, most, 16, 5, "few")
        want = evict_ref(w, table, lens, 16, most // 3, 1, 2)
        w, table, lens = (torch.from_numpy(x).cuda() for x in (w, table, lens))
        freed, count = torch.empty_like(table), torch.empty_like(lens)
        given = table.clone()
        rc = lib.dilated_attn_evict_pages(*(t.data_ptr() for t in (w, table, lens, table, freed, count)), B, w.numel(), 16,
                                          most, most // 3, 1, 2, None)
        torch.cuda.synchronize()
        assert rc == 0 and all(np.array_equal(g.cpu().numpy(), x) for g, x in zip((table, freed, count), want))
        for more in (dict(keep=2 ** 64), dict(keep=0, first=2 ** 70), dict(keep=0, last=2 ** 64)):
            held, _, none = evict_pages(w, given, lens, 16, **more)
            assert torch.equal(held, given) and not bool(none.any())
