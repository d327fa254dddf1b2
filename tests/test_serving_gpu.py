"""The attention layer with normed heads, trained, and served from a paged cache.

Bars: the layer's gradients with head norms as the layer's without (3e-2 of each
gradient's largest entry, bf16); step against forward 4e-2 on outputs of size
about 1 (both round every intermediate to bf16, xPos about different centres),
1e-4 in float32."""
import numpy as np
import pytest
import torch

import workloads
from oracle.paged_ref import heads_ref
from oracle.dilated_ref import dilated_attention_ref
from tests.gpu_util import note, require_gpu, to64

pytestmark = pytest.mark.gpu
PATS = [(64, 1), (256, 3)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make(dtype, qk_norm, use_xpos=True, E=256, H=4):
    from paper_2307_02486_amd.layer import LongNetAttention
    torch.manual_seed(7)
    layer = LongNetAttention(E, H, PATS, device="cuda", dtype=dtype, qk_norm=qk_norm, use_xpos=use_xpos)
    if qk_norm:
        with torch.no_grad():
            layer.q_norm.add_(0.2 * torch.randn_like(layer.q_norm))
            layer.k_norm.add_(0.2 * torch.randn_like(layer.k_norm))
    return layer


def layer_oracle(x, p, H):
    """The layer's forward with head norms in float64."""
    def ln(t, g, b):
        m = t.mean(-1, keepdims=True)
        return (t - m) / np.sqrt(((t - m) ** 2).mean(-1, keepdims=True) + 1e-5) * g + b
    B, N, E = x.shape
    u = ln(x, p["ln_in_g"], p["ln_in_b"])
    q, k, v = ((u @ p["w" + n].T + p["b" + n]).reshape(B, N, H, E // H) for n in "qkv")
    pos = np.arange(N)
    q, k = heads_ref(q, p["q_norm"], pos, 1, N // 2), heads_ref(k, p["k_norm"], pos, -1, N // 2)
    a, _ = dilated_attention_ref(q, k, v, PATS, True)
    return ln(a.reshape(B, N, E), p["ln_sub_g"], p["ln_sub_b"]) @ p["wo"].T + p["bo"]


@pytest.mark.parametrize("dtype, bar", [(torch.float32, 1e-4), (torch.bfloat16, 4e-2)], ids=str)
def test_layer_with_head_norms_forward(dtype, bar):
    note(f"[serving] layer {dtype}")
    layer = make(dtype, True)
    x = workloads.make_random((2, 200, 256), dtype, 1.0, 5, "cuda", 0)
    with torch.no_grad():
        plain = layer(x)
    recorded = layer(x) if dtype == torch.bfloat16 else plain
    want = layer_oracle(to64(x), layer.float64_params(), 4)
    assert np.abs(to64(plain) - want).max() <= bar
    assert torch.equal(plain, recorded)


def test_layer_with_head_norms_gradients():
    """Against differences of the float64 oracle along random directions."""
    note("[serving] layer gradients")
    layer = make(torch.bfloat16, True)
    x = workloads.make_random((1, 130, 256), torch.bfloat16, 1.0, 6, "cuda", 0).requires_grad_()
    dy = workloads.make_random((1, 130, 256), torch.bfloat16, 1.0, 6, "cuda", 1)
    layer(x).backward(dy)
    p, x64, dy64 = layer.float64_params(), to64(x), to64(dy)
    rng = np.random.default_rng(0)
    got = {"q_norm": layer.q_norm.grad, "k_norm": layer.k_norm.grad, "x": x.grad, "wq": layer.q_proj.weight.grad}
    for key, grad in got.items():
        g = to64(grad)
        for _ in range(3):
            e = rng.normal(size=g.shape)

            def loss(h):
                at = dict(p)
                if key != "x":
                    at[key] = p[key] + h * e
                return (layer_oracle(x64 + h * e if key == "x" else x64, at, 4) * dy64).sum()
            num = (loss(1e-5) - loss(-1e-5)) / 2e-5
            # the error of a sum of n independent errors of at most 3e-2 max|g| each, three deviations
            assert abs(num - (g * e).sum()) <= 3 * 3e-2 * np.abs(g).max() * np.sqrt(e.size), key


@pytest.mark.parametrize("dtype, bar", [(torch.float32, 1e-4), (torch.bfloat16, 4e-2)], ids=str)
@pytest.mark.parametrize("qk_norm, use_xpos", [(False, True), (True, True), (False, False)], ids=str)
def test_step_gives_the_rows_of_forward(dtype, bar, qk_norm, use_xpos):
    """Three sequences served together: prompts in chunks, then token by token."""
    from paper_2307_02486_amd.serving import PagedCache
    note(f"[serving] step {dtype} {qk_norm} {use_xpos}")
    layer = make(dtype, qk_norm, use_xpos)
    lengths = {"a": 150, "b": 41, "c": 7}
    xs = {s: workloads.make_random((n, 256), dtype, 1.0, 9, "cuda", t) for t, (s, n) in enumerate(lengths.items())}
    with torch.no_grad():
        want = {s: layer(x[None])[0] for s, x in xs.items()}
    cache = PagedCache(40, 16, 12, 4, 64, device="cuda", dtype=dtype)
    done = {s: 0 for s in xs}
    steps = [(["a", "b"], [100, 30]), (["c", "a", "b"], [2, 46, 8]), (["b", "a", "c"], [1, 1, 1]), (["a"], [1]),
             (["b", "a", "c"], [2, 2, 4])]
    for names, new in steps:
        batch = cache.extend(names, new)
        y = layer.step(torch.cat([xs[s][done[s]: done[s] + n] for s, n in zip(names, new)]), cache, batch)
        at = 0
        for s, n in zip(names, new):
            err = float((y[at: at + n].float() - want[s][done[s]: done[s] + n].float()).abs().max())
            assert err <= bar, (names, new, s, err)
            done[s] += n
            at += n
    assert done == lengths
    cache.release("a")
    batch = cache.extend(["d"], [20])  # pages that others have used before
    y = layer.step(xs["b"][:20], cache, batch)
    assert float((y.float() - want["b"][:20].float()).abs().max()) <= bar
