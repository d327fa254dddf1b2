"""Eviction in launches of rows: from 2^24 workgroups on a launch is a grid of rows of
2^20 of them, with workgroups past its end, which have no sequence."""
import pytest
import torch

from tests.gpu_util import note, require_gpu

pytestmark = pytest.mark.gpu
GUARD = 0x5A5A5A5A


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def evict(weights, table, lens, out, freed, count, B, page, most, keep, first, last):
    from paper_2307_02486_amd import _lib
    rc = _lib.load().dilated_attn_evict_pages(*(t.data_ptr() for t in (weights, table, lens, out, freed, count)), B,
                                              weights.numel(), page, most, keep, first, last, None)
    torch.cuda.synchronize()
    assert rc == 0


def test_sequences_past_the_end_of_the_launch_are_not_there():
    """2^24 + 1 tables of a page each: the last row of the launch has 2^20 - 1
    workgroups too many, and behind the outputs is other memory."""
    note("[evict] 2^24 + 1 tables")
    B, behind = (1 << 24) + 1, 1 << 20
    table = torch.arange(B + behind, dtype=torch.int32, device="cuda")
    lens = torch.ones(B + behind, dtype=torch.int32, device="cuda")
    weights = torch.rand(B + behind, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    lens[::3] = 0
    out, freed, count = (torch.full((B + behind,), GUARD, dtype=torch.int32, device="cuda") for _ in range(3))
    evict(weights, table, lens, out, freed, count, B, 16, 1, 0, 0, 0)
    goes = lens[:B] > 0
    gone = torch.full_like(table[:B], -1)
    assert torch.equal(count[:B], goes.int())
    assert torch.equal(out[:B], torch.where(goes, gone, table[:B]))
    assert torch.equal(freed[:B], torch.where(goes, table[:B], gone))
    for t in (out, freed, count):
        assert bool((t[B:] == GUARD).all())
