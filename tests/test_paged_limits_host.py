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


PAPER = ((2048, 1), (4096, 2), (8192, 4), (16384, 6), (32768, 12))


def test_the_weights_workspace_goes_by_the_segments_not_by_the_table():
    """A row's sums are those of pages that its patterns reach: a wider table needs no
    more, once it holds them."""
    for T, B in ((1, 1), (64, 64), (1087, 64), (8255, 64)):
        sizes = dict(T=T, B=B, H=32, Hkv=8, D=128, num_pages=1 << 16, patterns=PAPER)
        got = [weights_need(max_pages=n, **sizes) for n in (4096, 8192, 65536, 1 << 20)]
        assert got[0] == got[1] == got[2] == got[3]
    # one token: a page more than a segment's at either end, of each pattern and head, in lines of 128 bytes
    each = 4 * sum(w // 16 + 2 for w, _ in PAPER)
    assert each <= weights_need(T=1, B=1, H=1, Hkv=1, max_pages=65536, patterns=PAPER) <= each + 5 * 256
    assert 4 * 5 * 8 <= weights_need(T=1, B=1, H=1, Hkv=1, max_pages=8, patterns=PAPER) <= 5 * 128
    # 64 sequences, 4096 new tokens of one: no more than the attention of the call
    sizes = dict(T=4159, B=64, H=12, Hkv=12, D=64, num_pages=1 << 16, patterns=PAPER, max_pages=65536)
    assert weights_need(**sizes) <= 2 * need(**sizes)
