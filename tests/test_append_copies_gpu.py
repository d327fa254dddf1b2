"""The append without norm and rotation is a copy."""
import numpy as np
import pytest
import torch

import workloads
from tests.gpu_util import note, require_gpu
from tests.test_heads_gpu import paged

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_append_without_rotation_or_norm_copies(dtype):
    """Queries and keys are then what they were, infinities and the largest values too."""
    from paper_2307_02486_amd import cache_append
    note(f"[append] copies {dtype}")
    new, page, H, Hkv, D = [5, 40], 16, 4, 2, 64
    table, lens, start, dev, pages = paged(new, [3, 0], page)
    q, k, v = (workloads.make_random((45, h, D), dtype, 1.0, 95, "cuda", t) for t, h in enumerate((H, Hkv, Hkv)))
    big = torch.finfo(dtype).max
    for x in (q, k, v):
        x[::3, :, 7], x[1::4, :, 8], x[2::5, :, 20], x[::2, :, 33] = float("inf"), float("-inf"), big, -big
    kc, vc = (torch.zeros((pages, Hkv, page, D), dtype=dtype, device="cuda") for _ in range(2))
    qo = cache_append(q, k, v, kc, vc, *dev, rotate=False)
    torch.cuda.synchronize()
    assert torch.equal(qo, q)
    for b in range(2):
        pos = np.arange(lens[b] - new[b], lens[b])
        p, s = torch.from_numpy(table[b, pos // page]).long().cuda(), torch.from_numpy(pos % page).cuda()
        rows = slice(int(start[b]), int(start[b + 1]))
        assert torch.equal(kc[p, :, s], k[rows]) and torch.equal(vc[p, :, s], v[rows])
