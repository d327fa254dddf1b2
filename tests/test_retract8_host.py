"""A batch taken back from a cache in 8 bits whose append had run, with the append of the
reference: the blocks' earlier values and scales are as they were.  No GPU."""
import numpy as np
import pytest
import torch

from tests.cache8 import append_ref, bytes_of, unscaled

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
HKV, D = 2, 32


def make(page=16, layers=2, **change):
    from paper_2307_02486_amd.serving import PagedCache
    cache = PagedCache(24, page, 8, HKV, D, layers=layers, device="cpu", dtype=F8, **change)
    for c in (*cache.k, *cache.v, *cache.k_scale, *cache.v_scale):
        c.view(torch.uint8).fill_(100)
    return cache


def append(cache, batch, x, layers=None):
    """New rows x [T, HKV, D] as keys, twice as large as values, into these layers (default: all)."""
    table, lens, start = (t.numpy() for t in batch[:3])
    for i in range(len(cache.k)) if layers is None else layers:
        for c, s, mul in ((cache.k[i], cache.k_scale[i], 1.0 + i), (cache.v[i], cache.v_scale[i], 2.0)):
            vals, exps = unscaled(c), bytes_of(s).astype(np.int64) - 127
            append_ref(vals, exps, table, lens, start, x * mul, cache.page_size)
            c.copy_(torch.from_numpy(vals).float().to(F8))
            s.view(torch.uint8).copy_(torch.from_numpy((exps + 127).astype(np.uint8)))


def rows(seed, n, size=1.0):
    return np.random.default_rng(seed).normal(size=(n, HKV, D)) * size


def held(cache, sequence):
    """The bytes of a sequence's rows and the scales of its blocks, of all layers."""
    n, size = cache.length(sequence), min(cache.page_size, 16)
    pages, out = cache._pages[sequence], []
    for c in (*cache.k, *cache.v):
        out.append(np.concatenate([bytes_of(c)[p] for p in pages], axis=1)[:, :n])
    for s in (*cache.k_scale, *cache.v_scale):
        out.append(np.concatenate([bytes_of(s)[p] for p in pages], axis=1)[:, : -(-n // size)])
    return out


def equal(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b)) and len(a) == len(b)


@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("size", [0.1, 30.0, 1e30])
@pytest.mark.parametrize("ran", [None, [1], []], ids=["all layers", "one layer", "no layer"])
def test_earlier_values_are_as_they_were(page, size, ran):
    cache = make(page)
    append(cache, cache.extend(["a", "b", "c"], [13, 16, 5]), rows(1, 34))
    for s in cache.k_scale:  # a NaN, which stays one
        assert s.shape == (24, HKV, max(page // 16, 1))
    cache.k[0].view(torch.uint8)[cache._pages["a"][12 // page], 0, 12 % page, 3] = 0x7F
    cache.k[0].view(torch.uint8)[cache._pages["a"][12 // page], 0, 12 % page, 4] = 0x80
    before = {s: held(cache, s) for s in "abc"}
    for names, new in ((["a", "b", "c"], [1, 1, 1]), (["c"], [20]), (["b", "a"], [3, 0])):
        batch = cache.extend(names, new)
        append(cache, batch, rows(2, sum(new), size), ran)
        cache.retract(batch)
        assert all(equal(held(cache, s), before[s]) for s in "abc")
    assert not cache._before


def test_a_batch_made_before_the_one_before_it_ran():
    """Two steps extended ahead of their layers: taking the second back leaves the
    first one's values, rescaled where the second has rescaled them."""
    cache = make()
    append(cache, cache.extend(["a"], [5]), rows(3, 5))
    one, two = cache.extend(["a"], [4]), cache.extend(["a"], [2])
    append(cache, one, rows(4, 4))
    append(cache, two, rows(5, 2, 300.0))
    after = held(cache, "a")
    cache.retract(two)
    assert cache.length("a") == 9
    n = [c[:, :9] for c in after[:4]] + after[4:]
    assert equal(held(cache, "a"), n)


def test_what_is_kept_goes_with_the_batch(monkeypatch):
    cache = make(weigh=True)
    one = cache.extend(["a", "b"], [5, 7])
    assert not cache._before  # no block with earlier tokens
    two = cache.extend(["a", "b"], [1, 1])
    assert list(cache._before) == [two.number]
    three = cache.extend(["a"], [1])  # two cannot be taken back any more
    assert list(cache._before) == [three.number]
    with pytest.raises(ValueError):
        cache.retract(two)
    four = cache.extend(["b"], [9])
    assert sorted(cache._before) == [three.number, four.number]
    cache.release("b")
    assert list(cache._before) == [three.number]
    from oracle.compressed_ref import evict_ref
    from paper_2307_02486_amd import serving

    def evict(weights, table, lens, page, keep, first, last):
        got = evict_ref(weights.numpy(), table.numpy(), lens.numpy(), page, keep, first, last)
        return tuple(torch.from_numpy(x) for x in got)

    monkeypatch.setattr(serving, "evict_pages", evict)
    five = cache.extend(["a"], [41])
    assert list(cache._before) == [five.number]
    assert cache.evict(1, ["a"], first=0, last=1) == 2 and not cache._before
    six = cache.extend(["a"], [16])  # 48 held: a block of its own
    assert not cache._before and cache.length("a") == 64
    cache.retract(six)
    assert one.max_new == 7 and cache.length("a") == 48


def test_wide_caches_keep_nothing():
    from paper_2307_02486_amd.serving import PagedCache
    cache = PagedCache(6, 16, 4, HKV, D, device="cpu")
    cache.extend(["a"], [5])
    batch = cache.extend(["a"], [1])
    assert not cache._before
    cache.retract(batch)
    assert cache.length("a") == 5


def test_a_cache_made_in_inference_mode_serves_outside():
    for inside in (True, False):
        with torch.inference_mode(not inside):
            cache = make(weigh=True)
        with torch.inference_mode(inside):
            append(cache, cache.extend(["a"], [5]), rows(6, 5))
            before = held(cache, "a")
            batch = cache.extend(["a"], [1])
            append(cache, batch, rows(7, 1, 100.0))
            cache.retract(batch)
            assert equal(held(cache, "a"), before)
