"""Steps of a layer pair over a cache in 8 bits, eager and replayed: the same bytes of
values and scales; and a step taken back whose append had rescaled blocks: what came
before and what comes after are as if it had not run."""
import pytest
import torch

import workloads
from tests.cache8 import F8
from tests.gpu_util import note, require_gpu
from tests.test_serving_gpu import make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def caches(cache):
    return (*cache.k, *cache.v, *cache.k_scale, *cache.v_scale)


def serve(dtype, captured, taken_back, steps=9):
    """(outputs, cache, bytes that the step taken back changed, and how many of them are so after it)."""
    from paper_2307_02486_amd.serving import Batch, PagedCache
    layers = [make(dtype, True), make(dtype, False)]
    cache = PagedCache(20, 16, 8, 4, 64, layers=2, device="cuda", dtype=F8, weigh=True)
    for c in caches(cache):
        c.view(torch.uint8).zero_()

    def run(x, batch):
        for i, layer in enumerate(layers):
            x = layer.step(x, cache, batch, i)
        return x

    x = workloads.make_random((61, 256), dtype, 1.0, 3, "cuda", 0)
    outs, graph, rounded = [run(x, cache.extend(["a", "b"], [40, 21]))], None, (0, 0)
    for t in range(steps):
        for back in ([True, False] if t == taken_back else [False]):
            batch = cache.extend(["a", "b"], [1, 1])
            x = workloads.make_random((2, 256), dtype, 1.0, 20 + t, "cuda", 0)
            if graph is None and captured:
                fixed_x, fixed = x.clone(), Batch(*(b.clone() for b in batch[:3]), 1)
                saved, had = [c.view(torch.uint8).clone() for c in caches(cache)], cache.weights.clone()
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):  # once beforehand, then as it was
                    run(fixed_x, fixed)
                torch.cuda.current_stream().wait_stream(side)
                for c, s in zip(caches(cache), saved):
                    c.view(torch.uint8).copy_(s)
                cache.weights.copy_(had)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    held = run(fixed_x, fixed)
            if back:  # keys and values 64 times as large
                was = [c.view(torch.uint8).clone() for c in caches(cache)]
                had = cache.weights.clone()
                for layer in layers:
                    for m in (layer.k_proj, layer.v_proj):
                        m.weight.data.mul_(64)
            if captured:
                for s, n in zip((fixed_x, *fixed[:3]), (x, *batch[:3])):
                    s.copy_(n)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                y = held.clone()
            else:
                y = run(x, batch)
            if not back:
                outs.append(y)
                continue
            for layer in layers:
                for m in (layer.k_proj, layer.v_proj):
                    m.weight.data.mul_(1 / 64)
            changed = [a != c.view(torch.uint8) for a, c in zip(was, caches(cache))]
            cache.retract(batch)
            after = [a != c.view(torch.uint8) for a, c in zip(was, caches(cache))]
            cache.weights.copy_(had)
            rounded = sum(int(x.sum()) for x in changed), sum(int(x.sum()) for x in after)
            new = 2 * 2 * 2 * 4 * 64  # the step's own rows: tokens, layers, keys and values, heads of 64
            assert rounded[0] > 2 * new >= 2 * rounded[1]
    return outs, cache


@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_a_step_taken_back_leaves_nothing(dtype, captured):
    note(f"[retract8] {dtype} captured={captured}")
    want, plain = serve(dtype, False, None)
    got, cache = serve(dtype, captured, 4)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and len(want) == len(got)
    for a, b in zip(caches(plain), caches(cache)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(plain.weights, cache.weights) and not cache._before.keys() - {cache._number}


@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_replayed_steps_write_the_values_and_scales_of_eager_ones(dtype):
    note(f"[retract8] replays {dtype}")
    want, eager = serve(dtype, False, None)
    got, replayed = serve(dtype, True, None)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for a, b in zip(caches(eager), caches(replayed)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(eager.weights, replayed.weights)
