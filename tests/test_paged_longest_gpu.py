"""A sequence of as many positions as a table may have, 2^31 - 2^16, almost all of
whose pages are gone: positions, key numbers and page numbers next to 2^31.

Bars as in test_paged8_gpu (attention) and test_page_weights_gpu (weights)."""
import numpy as np
import pytest
import torch

import workloads
from tests.cache8 import elements, normal_pool
from tests.gpu_util import note, require_gpu, to64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
MOST = (1 << 31) - (1 << 16)
NEAR = [(4096, 1), (1 << 20, 3)]
DENSE = [(1 << 40, 1)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def long_sequence(page, Hkv, D, pages):
    """(K, V, their scales, table, positions that are there, K and V there in float64)."""
    width = MOST // page
    rng = np.random.default_rng(page)
    near = rng.permutation((1 << 21) // page)[: pages // 2]  # in the last two million positions
    at = np.unique(np.concatenate([[0, 1, width - 1, width - 2, width - 4, width // 2], width - 1 - near,
                                   rng.integers(0, width, pages // 3)]))[:pages]
    at = np.unique(np.concatenate([at, [width - 1]]))
    kc, ks = normal_pool(len(at), Hkv, page, D, 1)
    vc, vs = normal_pool(len(at), Hkv, page, D, 2)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, torch.from_numpy(at).cuda()] = torch.arange(len(at), dtype=torch.int32, device="cuda")
    pos = (at[:, None] * page + np.arange(page)).reshape(-1)
    k, v = (elements(c, s).transpose(0, 2, 1, 3).reshape(-1, Hkv, D) for c, s in ((kc, ks), (vc, vs)))
    return kc, vc, ks, vs, table, pos, k, v


def expected(q, first, patterns, pos, k, v, pages):
    """out, lse [H, T] and the weights of the pool's pages, key by key."""
    T, H, D = q.shape
    group = H // k.shape[1]
    out, lse, got = np.zeros(q.shape), np.full((H, T), -np.inf), np.zeros((pages, len(pos) // pages))
    for i in range(T):
        p = first + i
        for h in range(H):
            c = np.zeros(len(pos))
            for w, r in patterns:
                if (p % w) % r == h % r:
                    c += (pos // w == p // w) & ((pos % w) % r == h % r) & (pos <= p)
            sel = np.flatnonzero(c)
            if sel.size:
                s = k[sel, h // group] @ q[i, h] * D ** -0.5
                e = c[sel] * np.exp(s - s.max())
                out[i, h], lse[h, i] = e @ v[sel, h // group] / e.sum(), s.max() + np.log(e.sum())
                np.add.at(got.reshape(-1), sel, e / e.sum())
    return out, lse, got.sum(1)


@pytest.mark.parametrize("page, new, patterns, dtype", [
    (16, 1, DENSE, BF), (16, 1, [*NEAR, *DENSE], BF), (16, 70, NEAR, BF), (16, 3, NEAR, F32),
    (1, 1, [((1 << 30) + 12345, 1)], BF),   # page numbers next to 2^31, too
], ids=str)
def test_attention_and_weights_at_the_end_of_the_longest_table(page, new, patterns, dtype):
    from paper_2307_02486_amd import page_weights, paged_attn
    note(f"[longest] page={page} new={new} {patterns} {dtype}")
    H, Hkv, D = (4, 2, 32) if page > 1 else (1, 1, 32)
    kc, vc, ks, vs, table, pos, k, v = long_sequence(page, Hkv, D, 48)
    q = workloads.make_random((new, H, D), dtype, 1.0, 7, "cuda", 0)
    dev = [table, torch.tensor([MOST], dtype=torch.int32, device="cuda"),
           torch.tensor([0, new], dtype=torch.int32, device="cuda")]
    want, wl, weight = expected(to64(q), MOST - new, patterns, pos, k, v, kc.shape[0])
    out, lse = paged_attn(q, kc, vc, *dev, patterns, k_scale=ks, v_scale=vs, max_new=new)
    torch.cuda.synchronize()
    note("  attention done")
    to, tl = (5e-3, 1e-4) if dtype == BF else (2e-5, 1e-4)
    assert np.abs(to64(out) - want).max() <= to * np.abs(v).max()
    fin = np.isfinite(wl)
    assert np.array_equal(np.isneginf(to64(lse)), ~fin) and np.abs(to64(lse)[fin] - wl[fin]).max() <= tl
    exact = torch.from_numpy(wl.astype(np.float32)).cuda()
    for hint in (new, 0):
        weights = torch.zeros(kc.shape[0], device="cuda")
        page_weights(q, exact, kc, ks, *dev, patterns, weights, max_new=hint)
        torch.cuda.synchronize()
        note("  weights done")
        assert (np.abs(to64(weights) - weight) <= 2e-5 * weight + 1e-6).all()
