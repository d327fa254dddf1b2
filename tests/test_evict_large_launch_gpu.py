"""Eviction in launches of rows: from 2^32 work-items on (2^24 workgroups of 256 threads,
2^22 of 1024) a launch is a grid of rows of 2^20 workgroups, with some past its end,
which have no sequence."""
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


def test_every_sequence_of_a_launch_of_large_workgroups():
    """2^22 + 3 tables of 1025 pages, beyond what four waves list, in place: 17 GB, of
    which a few rows name pages, the last three among them."""
    note("[evict] 2^22 + 3 tables of 1025 pages")
    B, most, page, pool = (1 << 22) + 3, 1025, 4, 40
    table = torch.full((B, most), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    count, freed = torch.full_like(lens, GUARD), torch.full_like(table, GUARD)
    weights = torch.arange(pool, dtype=torch.float32, device="cuda").flip(0).contiguous()  # the last pages go first
    rows = [0, 1, (1 << 20) + 5, (1 << 22) - 1, 1 << 22, B - 2, B - 1]
    lens[rows] = most * page
    for r in rows:
        table[r, 1000: 1005] = torch.arange(5, dtype=torch.int32, device="cuda") + r % 7
    evict(weights, table, lens, table, freed, count, B, page, most, 2, 0, 0)
    assert int((count != 0).sum()) == len(rows)
    for r in rows:
        assert int(count[r]) == 3
        assert freed[r, :3].tolist() == [r % 7 + 2, r % 7 + 3, r % 7 + 4]
        assert table[r, 1000: 1005].tolist() == [r % 7, r % 7 + 1, -1, -1, -1]
    assert sum(int((freed[r0: r0 + (1 << 20)] != -1).sum()) for r0 in range(0, B, 1 << 20)) == 3 * len(rows)
    assert sum(int((table[r0: r0 + (1 << 20)] != -1).sum()) for r0 in range(0, B, 1 << 20)) == 2 * len(rows)
