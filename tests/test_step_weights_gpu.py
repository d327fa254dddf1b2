"""The weights that steps add to their cache's pages, from the very queries of the steps.

Bar: an lse of the attention is within 1e-4 of float64's, so a pair's weight within 1e-4 of
itself, and page_weights within 2e-5 (test_page_weights_gpu)."""
import numpy as np
import pytest
import torch

import workloads
from tests.cache8 import F8
from tests.gpu_util import note, require_gpu, to64
from tests.test_page_weights_gpu import reference
from tests.test_paged8_gpu import held_values
from tests.test_serving_gpu import PATS, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_steps_add_what_their_tokens_give(dtype, monkeypatch):
    from paper_2307_02486_amd import layer as module
    from paper_2307_02486_amd.serving import PagedCache
    note(f"[step weights] {dtype}")
    seen = []

    def recorded(q, lse, k_cache, k_scale, table, lens, start, patterns, weights, **more):
        seen.append((q.clone(), weights.clone(), [t.cpu().numpy() for t in (table, lens, start)]))
        return page_weights(q, lse, k_cache, k_scale, table, lens, start, patterns, weights, **more)

    page_weights = module.page_weights
    monkeypatch.setattr(module, "page_weights", recorded)
    layers = [make(dtype, True), make(dtype, False)]
    cache = PagedCache(40, 16, 12, 4, 64, layers=2, device="cuda", dtype=F8, weigh=True)
    for c in (*cache.k, *cache.v):  # what no sequence holds is NaN
        c.view(torch.uint8).fill_(0x7F)
    for s in (*cache.k_scale, *cache.v_scale):
        s.view(torch.uint8).fill_(127)
    for t, (names, new) in enumerate(((["a", "b"], [100, 30]), (["c", "a", "b"], [2, 46, 8]), (["b", "a", "c"], [1, 1, 1]))):
        batch = cache.extend(names, new)
        x = workloads.make_random((sum(new), 256), dtype, 1.0, 9 + t, "cuda", 0)
        for i, layer in enumerate(layers):
            x = layer.step(x, cache, batch, i)
            q, before, (table, lens, start) = seen.pop()
            pools = held_values(cache.k[i], cache.v[i], cache.k_scale[i], cache.v_scale[i])
            _, want = reference(q, pools, table, lens, start, 16, PATS)
            got = to64(cache.weights) - to64(before)
            assert (np.abs(got - want) <= 1.2e-4 * want + 1e-6 + 2.0 ** -23 * to64(cache.weights)).all()
            assert want.sum() > 0.9 * sum(new)  # a head of a token that sees a key gives one
        if t == 0:
            cache.evict(5, ["a"], first=1, last=1)
    assert not seen
