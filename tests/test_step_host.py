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
