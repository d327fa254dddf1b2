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
