"""What LongNetAttention.step refuses and answers before any kernel, and the
cache's book-keeping around it.  No GPU."""
import pytest
import torch

from paper_2307_02486_amd.layer import LongNetAttention
from paper_2307_02486_amd.serving import PagedCache


def make(**change):
    torch.manual_seed(3)
    args = dict(embed_dim=64, num_heads=2, patterns=[(8, 1), (16, 2)], device="cpu")
    args.update(change)
    return LongNetAttention(**args)


def cache_for(layer, num_pages=8, page_size=4, max_pages=4, **change):
    return PagedCache(num_pages, page_size, max_pages, layer.num_heads, layer.head_dim, device="cpu", **change)


def test_step_refuses_to_be_traced():
    """A trace would record empty outputs without the kernels that fill them."""
    layer = make()
    cache = cache_for(layer)
    batch = cache.extend(["a"], [3])
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="trace"):
        torch.jit.trace(lambda t: layer.step(t, cache, batch), (x,), check_trace=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_step_without_new_tokens(dtype):
    """No sequence has a new token: no rows in, none out."""
    layer = make(dtype=dtype)
    cache = cache_for(layer, dtype=dtype)
    batch = cache.extend(["a", "b"], [0, 0])
    y = layer.step(torch.zeros(0, 64, dtype=dtype), cache, batch)
    assert y.shape == (0, 64) and y.dtype == dtype


@pytest.mark.parametrize("shape", [(4, 64), (0, 64), (1, 5, 64), (64,), (5, 32)], ids=str)
def test_step_refuses_rows_that_are_not_the_batch_s_tokens(shape):
    """With fewer rows than new tokens the rest of the sequences would be read as
    the pool's memory was."""
    layer = make()
    cache = cache_for(layer)
    batch = cache.extend(["a", "b"], [3, 2])
    with pytest.raises(ValueError, match="5 new tokens"):
        layer.step(torch.zeros(shape, dtype=torch.bfloat16), cache, batch)


def test_batch_of_four_fields():
    """A batch that a caller puts together (tensors of a captured step, say) need
    not tell its tokens."""
    from paper_2307_02486_amd.serving import Batch
    i = torch.zeros(1, dtype=torch.int32)
    batch = Batch(i[None], i, torch.zeros(2, dtype=torch.int32), 1)
    layer = make()
    assert layer.step(torch.zeros(0, 64, dtype=torch.bfloat16), cache_for(layer), batch).shape == (0, 64)


def append_accepts(reach, center, gamma, scale_base):
    """Whether the library's append takes a table of `reach` positions (no tokens: nothing is launched)."""
    from paper_2307_02486_amd import _lib
    lib = _lib.load()
    cache = _lib.PagedCacheArgs(0x1000000, 0x8000000, 0x3000000, 0x3100000, 0x3200000, 1, 1, reach)
    rc = lib.dilated_attn_cache_append(None, None, None, None, None, None, cache, 0, 1, 2, 2, 32, 64, 64, 64, 0.0, 1,
                                       center, 10000.0, gamma, scale_base, 1, None)
    assert _lib.ERRORS[rc] in ("DA_OK", "DA_EINVAL")
    return rc == 0


@pytest.mark.parametrize("gamma, scale_base", [(0.4, 512.0), (0.4, 37.5), (2.0, 100.0), (0.1, 8192.0), (0.7, 0.3)])
def test_the_reach_of_xpos_is_the_library_s(gamma, scale_base):
    from paper_2307_02486_amd.serving import xpos_span
    span = xpos_span(gamma, scale_base)
    assert append_accepts(2 * span + 1, span, gamma, scale_base)
    assert not append_accepts(2 * span + 2, span, gamma, scale_base)
    assert not append_accepts(2 * span + 2, span + 1, gamma, scale_base)


def test_caches_beyond_the_reach_of_xpos():
    """With the layer's defaults a table of 566 pages of 64 is the largest: one
    more is refused before the pool is there, and by step for a cache that was
    not told of xPos; a layer without xPos takes any."""
    for pages in (567, 1024):
        with pytest.raises(ValueError, match="36261 positions"):
            PagedCache(4, 64, pages, 2, 32, device="cpu", xpos=(0.4, 512.0))
    for center in (-1, 64, 50):
        with pytest.raises(ValueError, match="centre"):
            PagedCache(4, 8, 8, 2, 32, device="cpu", center=center, xpos=(0.4, 1.0))
    assert PagedCache(4, 64, 566, 2, 32, device="cpu", xpos=(0.4, 512.0)).center == 566 * 32
    layer = make()
    cache = cache_for(layer, page_size=64, max_pages=567)
    batch = cache.extend(["a"], [1])
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="36261 positions"):
        layer.step(x, cache, batch)
    with pytest.raises(RuntimeError, match="GPU only"):  # past this check
        make(use_xpos=False, dtype=torch.float32).step(x.float(), cache, batch)
    cache = cache_for(layer, page_size=64, max_pages=566)
    with pytest.raises(RuntimeError, match="GPU only"):
        make(dtype=torch.float32).step(x.float(), cache, cache.extend(["a"], [1]))


def state(cache):
    return {s: (cache.length(s), tuple(p)) for s, p in cache._pages.items()}, sorted(cache._free)


def test_a_batch_whose_step_failed_is_taken_back():
    """Lengths and pages are as before extend: the next step does not attend to
    tokens that were never written."""
    layer = make()
    cache = cache_for(layer)
    cache.extend(["a", "b"], [5, 4])
    before = state(cache)
    batch = cache.extend(["b", "new", "a"], [5, 6, 0])
    assert cache.length("new") == 6 and cache.length("b") == 9
    with pytest.raises(ValueError):
        layer.step(torch.zeros(3, 64, dtype=torch.bfloat16), cache, batch)
    cache.retract(batch)
    assert state(cache) == before and cache.length("new") == 0
    with pytest.raises(ValueError):
        cache.retract(batch)  # once
    later = cache.extend(["b"], [1])
    assert later.seq_lens.tolist() == [5]
    batch = cache.extend(["b"], [2])
    cache.extend(["b"], [1])
    after = state(cache)
    with pytest.raises(ValueError):
        cache.retract(batch)  # others came since
    cache.release("a")
    with pytest.raises(ValueError):
        cache.retract(later._replace(sequences=("b", "a"), new=(1, 1)))
    assert state(cache)[0]["b"] == after[0]["b"]


def test_only_whole_batches_are_taken_back():
    from paper_2307_02486_amd.serving import Batch
    cache = cache_for(make())
    cache.extend(["a"], [3])
    one = cache.extend(["a", "b"], [1, 2])
    cache.release("b")
    before = state(cache)
    with pytest.raises(ValueError):
        cache.retract(one)
    assert state(cache) == before
    with pytest.raises(ValueError):
        cache.retract(Batch(one.block_table, one.seq_lens, one.q_start, 1))


def test_a_sequence_of_the_same_name_and_length_is_another():
    cache = cache_for(make())
    batch = cache.extend(["a"], [3])
    cache.release("a")
    cache.extend(["a"], [3])
    with pytest.raises(ValueError):
        cache.retract(batch)
    assert cache.length("a") == 3
