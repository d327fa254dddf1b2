"""The page weights' workspace, of just the bytes that are asked for, between guards: rows
deep in long sequences, several segments of a chunk, tables far wider than the patterns."""
import numpy as np
import pytest
import torch

from tests.gpu_util import note, require_gpu, to64
from tests.test_page_weights_gpu import reference
from tests.test_paged8_gpu import held_values, setup

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("new, before, H, Hkv, D, page, patterns, dtype", [
    ([1, 1, 1], [900, 31, 700], 12, 4, 64, 16, [(64, 1), (256, 3), (100, 5)], BF),
    ([3, 2, 0, 0, 1, 0], [500, 65, 7, 0, 129, 1], 8, 2, 32, 1, [(33, 1), (128, 2)], BF),
    ([157, 1, 40], [600, 1000, 3], 4, 2, 64, 8, [(50, 1), (128, 3), (1 << 20, 7)], BF),
    ([64], [1500], 4, 4, 128, 64, [(70, 1), (100, 2)], BF),
    ([9, 70], [300, 511], 6, 2, 32, 16, [(512, 1), (600, 3), (16, 1)], F32),
], ids=str)
@pytest.mark.parametrize("wider", [1, 700])
def test_no_more_is_written_than_was_asked_for(new, before, H, Hkv, D, page, patterns, dtype, wider):
    from paper_2307_02486_amd import page_weights, page_weights_workspace_bytes
    note(f"[weights] workspace {new} {before} page={page} wider={wider}")
    q, kc, vc, ks, vs, dev, table, lens, start = setup(new, before, H, Hkv, D, page, dtype)
    table = np.concatenate([table, np.full((len(new), wider), -1, np.int32)], axis=1)
    dev[0] = torch.from_numpy(table).cuda()
    lse64, want = reference(q, held_values(kc, vc, ks, vs), table, lens, start, page, patterns)
    lse = torch.from_numpy(lse64.T.astype(np.float32)).contiguous().cuda()
    for hint in (None, max(new)):
        need = page_weights_workspace_bytes(q.shape[0], len(new), H, Hkv, D, kc.shape[0], page, table.shape[1], patterns,
                                            dtype, hint)
        guard = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        weights = torch.zeros(kc.shape[0], device="cuda")
        page_weights(q, lse, kc, ks, *dev, patterns, weights, workspace=guard[4096: 4096 + need], max_new=hint)
        torch.cuda.synchronize()
        assert bool((guard[:4096] == 0x5A).all()) and bool((guard[4096 + need:] == 0x5A).all())
        assert (np.abs(to64(weights) - want) <= 2e-5 * want + 1e-6).all()
