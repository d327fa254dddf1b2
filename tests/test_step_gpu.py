"""The serving step over several layers and in a graph, and the trained layer with
normed heads element by element."""
import numpy as np
import pytest
import torch

import workloads
from tests.gpu_util import note, require_gpu, to64

pytestmark = pytest.mark.gpu
PATS = [(64, 1), (256, 3)]
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make(dtype, seed=7, qk_norm=True):
    from paper_2307_02486_amd.layer import LongNetAttention
    torch.manual_seed(seed)
    layer = LongNetAttention(256, 4, PATS, device="cuda", dtype=dtype, qk_norm=qk_norm)
    if qk_norm:
        with torch.no_grad():
            layer.q_norm.add_(0.2 * torch.randn_like(layer.q_norm))
            layer.k_norm.add_(0.2 * torch.randn_like(layer.k_norm))
    return layer


def counts(N, H):
    """[H, N, N]: how many patterns let the query of a row see the key of a column."""
    p = torch.arange(N)
    c = torch.zeros(H, N, N, dtype=torch.float64)
    for w, r in PATS:
        for h in range(H):
            kept = (p % w) % r == h % r
            c[h] += (p[:, None] // w == p[None] // w) & kept[:, None] & kept[None] & (p[None] <= p[:, None])
    return c


def layer64(x, p, H):
    """The layer's forward in float64 torch operations, for autograd."""
    ln = torch.nn.functional.layer_norm
    B, N, E = x.shape
    D = E // H
    u = ln(x, (E,), p["ln_in_g"], p["ln_in_b"], 1e-5)
    q, k, v = ((u @ p["w" + n].T + p["b" + n]).view(B, N, H, D) for n in "qkv")
    i = torch.arange(D // 2, dtype=torch.float64)
    pos = torch.arange(N, dtype=torch.float64)[:, None]
    angle, zeta = pos * 10000.0 ** (-2 * i / D), (2 * i / D + 0.4) / 1.4

    def heads(t, w, sign):
        t = t / (t.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w
        s = zeta ** (sign * (pos - N // 2) / 512.0)
        c, n = (s * angle.cos())[:, None], (s * angle.sin())[:, None]
        return torch.stack((t[..., 0::2] * c - t[..., 1::2] * n, t[..., 0::2] * n + t[..., 1::2] * c), -1).flatten(-2)

    q, k = heads(q, p["q_norm"], 1), heads(k, p["k_norm"], -1)
    c = counts(N, H)
    s = (q.transpose(1, 2) @ k.transpose(1, 2).transpose(2, 3)) * D ** -0.5
    s = s.masked_fill(c == 0, -torch.inf)
    s = s - s.amax(-1, keepdim=True).clamp_min(-1e30).detach()
    e = s.exp() * c
    a = e / e.sum(-1, keepdim=True).clamp_min(1e-300) @ v.transpose(1, 2)
    a = a.transpose(1, 2).reshape(B, N, E)
    return ln(a, (E,), p["ln_sub_g"], p["ln_sub_b"], 1e-5) @ p["wo"].T + p["bo"]


NAMES = {"ln_in_g": "ln_in.weight", "ln_in_b": "ln_in.bias", "wq": "q_proj.weight", "bq": "q_proj.bias",
         "wk": "k_proj.weight", "bk": "k_proj.bias", "wv": "v_proj.weight", "bv": "v_proj.bias",
         "ln_sub_g": "ln_sub.weight", "ln_sub_b": "ln_sub.bias", "wo": "out_proj.weight", "bo": "out_proj.bias",
         "q_norm": "q_norm", "k_norm": "k_norm"}


# The bar of the layer without head norms: 3e-2 of a gradient's largest entry (the
# attention's backward is bf16's alone).  A bias of all keys moves a row's scores nearly alike, so
# its gradient is a sum of terms that cancel: it is held to the scale of q's bias's.
def test_gradients_with_head_norms_element_by_element():
    dtype, bar = BF, 3e-2
    note(f"[step] gradients {dtype}")
    layer = make(dtype)
    x = workloads.make_random((2, 130, 256), dtype, 1.0, 6, "cuda", 0).requires_grad_()
    dy = workloads.make_random((2, 130, 256), dtype, 1.0, 6, "cuda", 1)
    y = layer(x)
    y.backward(dy)
    p = {k: torch.from_numpy(v).requires_grad_() for k, v in layer.float64_params().items()}
    x64 = x.detach().cpu().double().requires_grad_()
    want = layer64(x64, p, 4)
    assert float((y.detach().cpu().double() - want.detach()).abs().max()) <= 4e-2
    want.backward(dy.cpu().double())
    params = dict(layer.named_parameters())
    got = {k: params[n].grad for k, n in NAMES.items()}
    assert set(got) == set(p)
    scale = {k: float(p[k].grad.abs().max()) for k in p}
    scale["bk"] = max(scale["bk"], scale["bq"])
    for k in p:
        err = float((got[k].cpu().double() - p[k].grad).abs().max())
        assert err <= bar * scale[k], f"{k}: {err / scale[k]:.2e}"
    assert float((x.grad.cpu().double() - x64.grad).abs().max()) <= bar * float(x64.grad.abs().max())


@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
def test_recorded_and_plain_forward_are_the_same(dtype):
    layer = make(dtype)
    x = workloads.make_random((2, 200, 256), dtype, 1.0, 5, "cuda", 0)
    with torch.no_grad():
        plain = layer(x)
    recorded = layer(x)
    assert recorded.requires_grad and torch.equal(plain, recorded.detach())


def serve(layers, xs, steps, cache, before=None):
    """The rows of every sequence through all layers, step by step."""
    done, rows = {s: 0 for s in xs}, {s: [] for s in xs}
    for names, new in steps:
        batch = cache.extend(names, new)
        y = torch.cat([xs[s][done[s]: done[s] + n] for s, n in zip(names, new)])
        for i, layer in enumerate(layers):
            y = y + layer.step(y, cache, batch, i)
        for s, part in zip(names, y.split(list(new))):
            rows[s].append(part)
            done[s] += part.shape[0]
    return {s: torch.cat(r) for s, r in rows.items()}


@pytest.mark.parametrize("dtype, bar", [(F32, 1e-4), (BF, 8e-2)], ids=str)
def test_step_through_two_layers(dtype, bar):
    """Each layer has its own keys in the same pages.  Bars: those of one layer,
    twice in bf16 (the second layer's input carries the first's error)."""
    from paper_2307_02486_amd.serving import PagedCache
    note(f"[step] two layers {dtype}")
    layers = [make(dtype, 7), make(dtype, 8, qk_norm=False)]
    xs = {s: workloads.make_random((n, 256), dtype, 1.0, 9, "cuda", t) for t, (s, n) in enumerate((("a", 90), ("b", 40)))}
    with torch.no_grad():
        want = {}
        for s, x in xs.items():
            y = x[None]
            for layer in layers:
                y = y + layer(y)
            want[s] = y[0]
    cache = PagedCache(20, 16, 8, 4, 64, layers=2, device="cuda", dtype=dtype, xpos=(0.4, 512.0))
    for pool in cache.k + cache.v:
        pool.fill_(float("nan"))
    got = serve(layers, xs, [(["a", "b"], [60, 3]), (["b", "a"], [36, 28]), (["a", "b"], [1, 1]), (["a"], [1])], cache)
    for s in xs:
        assert float((got[s].float() - want[s].float()).abs().max()) <= bar, s


@pytest.mark.parametrize("dtype, bar", [(F32, 1e-4), (BF, 4e-2)], ids=str)
def test_step_after_a_batch_taken_back_and_without_new_tokens(dtype, bar):
    from paper_2307_02486_amd.serving import PagedCache
    note(f"[step] taken back {dtype}")
    layer = make(dtype)
    x = workloads.make_random((50, 256), dtype, 1.0, 9, "cuda", 0)
    with torch.no_grad():
        want = layer(x[None])[0]
    cache = PagedCache(8, 16, 8, 4, 64, device="cuda", dtype=dtype)
    for pool in cache.k + cache.v:
        pool.fill_(float("nan"))
    y = [layer.step(x[:20], cache, cache.extend(["a"], [20]))]
    batch = cache.extend(["a"], [17])
    with pytest.raises(ValueError):
        layer.step(x[20:30], cache, batch)
    cache.retract(batch)
    y.append(layer.step(x[20:20], cache, cache.extend(["a"], [0])))
    y.append(layer.step(x[20:21], cache, cache.extend(["a"], [1])))
    y.append(layer.step(x[21:], cache, cache.extend(["a"], [29])))
    assert float((torch.cat(y).float() - want.float()).abs().max()) <= bar


def test_rows_past_the_batch_are_of_no_sequence():
    from paper_2307_02486_amd.serving import PagedCache
    layer = make(BF)
    x = workloads.make_random((9, 256), BF, 1.0, 9, "cuda", 0)
    caches = [PagedCache(8, 16, 8, 4, 64, device="cuda") for _ in range(2)]
    y, wide = (layer.step(x[:n], c, c.extend(["a", "b"], [3, 2])) for n, c in zip((5, 9), caches))
    assert float((wide[:5].float() - y.float()).abs().max()) <= 4e-2 and bool(torch.isfinite(wide.float()).all())
    for a, b in zip(caches[0].k + caches[0].v, caches[1].k + caches[1].v):
        pages = [caches[0]._pages[s][0] for s in ("a", "b")]
        assert torch.equal(a[pages[0], :, :3], b[pages[0], :, :3]) and torch.equal(a[pages[1], :, :2], b[pages[1], :, :2])


def test_captured_step():
    """A step of fixed tensors captured in a graph and replayed for the tokens that
    follow, with eager work between: every replay against the eager step."""
    from paper_2307_02486_amd.serving import Batch, PagedCache
    note("[step] graph")
    layer = make(BF)
    xs = workloads.make_random((2, 60, 256), BF, 1.0, 9, "cuda", 0)
    caches = [PagedCache(12, 16, 8, 4, 64, device="cuda") for _ in range(2)]
    for c in caches:
        layer.step(torch.cat([xs[0, :20], xs[1, :33]]), c, c.extend(["a", "b"], [20, 33]))
    lens = {"a": 20, "b": 33}
    first = caches[0].extend(["a", "b"], [1, 1])
    static = Batch(first.block_table.clone(), first.seq_lens.clone(), first.q_start.clone(), 1)
    x = torch.cat([xs[0, 20:21], xs[1, 33:34]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            layer.step(x, caches[0], static)  # writes the token's place; every replay does so again
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(x, caches[0], static)
    batch = first
    for i in range(5):
        at = [lens["a"] + i, lens["b"] + i]
        new = torch.stack([xs[0, at[0]], xs[1, at[1]]])
        if i:
            batch = caches[0].extend(["a", "b"], [1, 1])
        x.copy_(new)
        for t, s in zip(static[:3], batch[:3]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        want = layer.step(new, caches[1], caches[1].extend(["a", "b"], [1, 1]))
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
