"""The longest tables and the most sequences that the paged calls take: what their
kernels add to a position or a sequence's number has to fit 31 bits.  No GPU."""
import pytest
import torch

from tests.test_compressed_host import attend, lib, name, need as weights_need, weigh  # noqa: F401
from tests.test_paged_host import append, cache_args, need, paged_fwd

MOST = (1 << 31) - (1 << 16)
PAGES = [1, 2, 16, 1024, 1 << 15]


def plan_refuses(f, **sizes):
    from paper_2307_02486_amd import DilatedAttnError
    with pytest.raises(DilatedAttnError) as e:
        f(**sizes)
    return e.value.name


@pytest.mark.parametrize("page", PAGES)
def test_plans_of_the_longest_table(page):
    for f in (need, weights_need):
        assert f(T=1, B=1, page=page, max_pages=MOST // page) > 0
        assert plan_refuses(f, T=1, B=1, page=page, max_pages=MOST // page + 1) == "DA_EINVAL"
    assert need(T=1, B=1, page=1 << 16, max_pages=MOST >> 16) > 0


@pytest.mark.parametrize("page", PAGES)
def test_calls_refuse_a_longer_table(lib, page):  # noqa: F811
    longer = dict(num_pages=1, page_size=page, max_pages=MOST // page + 1)
    far = dict(q=None, qo=None, T=0, B=1, rotate=0, k=0, v=0)
    assert append(lib, cache=cache_args(**longer), **far) == "DA_EINVAL"
    assert append(lib, cache=cache_args(num_pages=1, page_size=page, max_pages=MOST // page), **far) == "DA_OK"
    assert paged_fwd(lib, T=0, B=1, cache=cache_args(**longer)) == "DA_EINVAL"
    assert attend(lib, T=0, B=1, **longer) == "DA_EINVAL" and weigh(lib, T=0, B=1, **longer) == "DA_EINVAL"
    pointers = (0x100, 0x1000000000, 0x3000000000, 0x4000000000, 0x6000000000, 0x8000000000)
    assert name(lib.dilated_attn_evict_pages(*pointers, 1, 10, page, MOST // page + 1, 1, 0, 0, None)) == "DA_EINVAL"


def test_calls_refuse_more_sequences(lib):  # noqa: F811
    for f in (need, weights_need):
        assert f(T=0, B=MOST, max_pages=1) >= 0
        assert plan_refuses(f, T=0, B=MOST + 1, max_pages=1) == "DA_EINVAL"
    assert paged_fwd(lib, T=0, B=MOST + 1) == "DA_EINVAL"
    assert append(lib, T=0, B=MOST + 1, q=0, qo=0, k=0, v=0) == "DA_EINVAL"


def test_weights_count_columns_in_blocks_of_tokens():
    """T * H just below 2^31, whose last block of 16 tokens would reach past it."""
    T = (1 << 15) - 2
    sizes = dict(T=T, B=1, H=1 << 16, Hkv=1, dtype=torch.bfloat16)
    assert plan_refuses(weights_need, **sizes) == "DA_EINVAL"  # H is below 2^16 anyway
    sizes["H"] = (1 << 16) - 1
    assert (T + 1) * sizes["H"] < 1 << 31 < (T + 32) * sizes["H"]
    assert plan_refuses(weights_need, **sizes) == "DA_EINVAL"
    assert weights_need(**dict(sizes, T=T - 64)) > 0
