"""Paged attention in launches of 2^24 workgroups and more, which are grids of rows
with workgroups past the launch's end.  (Those of the launch that steps through its
items did other workgroups' items once more: the same results, later.)"""
import numpy as np
import pytest
import torch

import workloads
from tests.gpu_util import note, require_gpu, to64
from tests.paged_rows import row

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def test_a_token_each_of_many_sequences_heads_and_patterns():
    from paper_2307_02486_amd import paged_attn
    note("[large launch] paged")
    B, H, D, page, width = 1025, 1024, 32, 16, 8   # 1025 * 1024 * 16 = 2^24 + 16384 items
    pats = [(64 + i, 1) for i in range(16)]
    pages = 24
    kc, vc = (workloads.make_random((pages, H, page, D), BF, 1.0, 31, "cuda", t) for t in (0, 1))
    q = workloads.make_random((B, H, D), BF, 1.0, 31, "cuda", 2)
    rng = np.random.default_rng(3)
    table = rng.integers(0, pages, (B, width)).astype(np.int32)  # sequences share pages: they are only read
    lens = rng.integers(1, width * page + 1, B).astype(np.int32)
    dev = [torch.from_numpy(x).cuda() for x in (table, lens, np.arange(B + 1, dtype=np.int32))]
    q32 = to64(q)

    def check(out, lse, tag):
        o64, l64 = to64(out), to64(lse)
        assert not np.isnan(o64).any() and np.isfinite(l64).all(), tag
        for b in (0, 1, 511, 512, B - 2, B - 1):
            at = np.arange(int(lens[b]))
            p = torch.from_numpy(table[b, at // page].astype(np.int64)).cuda()
            for h in (0, 1, 15, 16, H // 2, H - 1):
                k, v = (to64(c[p, h, torch.from_numpy(at % page).cuda()]) for c in (kc, vc))
                ro, rl, bar = row(q32[b, h], k, v, lens[b] - 1, h, pats)
                assert (np.abs(o64[b, h] - ro) <= bar).all() and abs(l64[h, b] - rl) <= 1e-4, (tag, b, h)

    for hint in (1, 5):  # every token by itself; as if a sequence could have five
        out = torch.full_like(q, float("nan"))
        out, lse = paged_attn(q, kc, vc, *dev, pats, max_new=hint, out=out)
        torch.cuda.synchronize()
        note(f"  hint {hint} done")
        check(out, lse, hint)
