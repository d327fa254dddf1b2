"""Host side of the compressed cache: refusals of the C ABI and of the binding, the
weights' plan, the cache's page keeping with pages that are gone, and the
references against the ones that are there.  No GPU."""
import numpy as np
import pytest
import torch

from oracle.compressed_ref import append_block, attention_ref, block_exponent, e4m3, evict_ref, key_weights_ref
from oracle.paged_ref import paged_attention_ref
from tests.test_paged_host import cache_args, name

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.fixture(scope="module")
def lib():
    from paper_2307_02486_amd import _lib
    return _lib.load()


def test_exports_the_declared_symbols(lib):
    for n in ("dilated_attn_cache_append_f8", "dilated_attn_paged_fwd_f8", "dilated_attn_page_weights_workspace",
              "dilated_attn_page_weights", "dilated_attn_evict_pages"):
        assert hasattr(lib, n)


# -- references ----------------------------------------------------------------
def test_e4m3_is_torch_s():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=4000) * np.exp2(rng.integers(-14, 7, 4000)), np.arange(-448, 449) / 2.0 ** 9,
                        np.arange(-448, 449), [2.0 ** -10, 3 * 2.0 ** -10, 464.0, 0.0]])
    x = x[np.abs(x) <= 464]
    want = torch.from_numpy(x).float().to(F8).double().numpy()
    assert np.array_equal(e4m3(np.float64(np.float32(x))), want)


def test_block_exponents():
    for amax, e in ((448.0, 0), (448.0001, 1), (1.75, -8), (1.76, -7), (1.0, -8), (0.0, -126), (2.0 ** -149, -126), (1e38, 118)):
        assert block_exponent(amax) == e, amax
    v, e = append_block(np.zeros((0, 2)), 99, np.array([[1.0, 0.3]]))
    assert e == -8 and np.array_equal(v, [[256.0, 80.0]])
    v, e = append_block(v, e, np.array([[100.0, np.inf]]))  # 400 lies between 12 and 13 times 32: to the even one
    assert e == -2 and np.array_equal(v[0], [4.0, 1.25]) and v[1, 0] == 384.0 and np.isnan(v[1, 1])


def test_references_with_all_pages_there():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(30, 2, 8)), rng.normal(size=(30, 2, 8))
    pats = [(8, 1), (16, 3)]
    out, lse = attention_ref(q, k, v, 25, pats, np.ones(30, bool))
    want, want_lse = paged_attention_ref(q, k, v, 25, pats)
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)
    w = key_weights_ref(q, k, 25, pats, np.ones(30, bool), lse)
    assert abs(w.sum() - np.isfinite(lse).sum()) < 1e-9


def test_evict_reference():
    w = np.array([5, 1, 3, 1, 9, 0], np.float32)
    table, freed, count = evict_ref(w, np.array([[0, 1, -1, 2, 3, 4, 77]], np.int32), [25], 4, 3, 1, 1)
    assert table.tolist() == [[0, -1, -1, 2, -1, 4, 77]] and freed[0, :3].tolist() == [1, 3, -1] and count[0] == 2


# -- the weights' plan -----------------------------------------------------------
def need(T=8, B=2, H=4, Hkv=2, D=64, num_pages=10, page=16, max_pages=4, patterns=((64, 1),), dtype=torch.bfloat16):
    from paper_2307_02486_amd import page_weights_workspace_bytes
    return page_weights_workspace_bytes(T, B, H, Hkv, D, num_pages, page, max_pages, patterns, dtype)


def test_workspace_holds_a_sum_of_each_unit_and_page():
    assert need() >= 2 * 2 * 4 * 4              # sequences, key heads, pages, floats
    assert need(patterns=((64, 2),)) >= 2 * 4 * 4 * 4  # both offsets of a key head
    assert need(T=2, patterns=((64, 2),), max_pages=64) < need(patterns=((64, 2),), max_pages=64)
    assert need(T=0) >= 0
    from paper_2307_02486_amd import page_weights_workspace_bytes
    sizes = (70, 80, 4, 2, 64, 100, 16, 64, ((64, 2),))  # a token's sums by themselves, or a sequence's
    assert len({page_weights_workspace_bytes(*sizes, max_new=n) for n in (None, 0, 1, 4)}) == 1
    assert page_weights_workspace_bytes(*sizes, max_new=70) != page_weights_workspace_bytes(*sizes)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(B=0), dict(H=0), dict(H=5), dict(Hkv=0), dict(num_pages=0), dict(page=12), dict(page=1 << 17),
    dict(max_pages=0), dict(max_pages=1 << 28), dict(patterns=()), dict(patterns=((4, 8),)), dict(patterns=((8, 1),) * 17),
    dict(T=1 << 30, H=1, Hkv=1, B=1 << 30, page=1, max_pages=(1 << 31) - 1),
], ids=str)
def test_plan_refuses(change):
    from paper_2307_02486_amd import DilatedAttnError
    with pytest.raises(DilatedAttnError) as e:
        need(**change)
    assert e.value.name == "DA_EINVAL"


# -- the C ABI, with pointers that are never followed ------------------------------
def f8_args(k_scale=0x5000000, v_scale=0x5100000, **change):
    from paper_2307_02486_amd import _lib
    return _lib.PagedCacheF8Args(cache_args(**change), k_scale, v_scale)


def append(lib, q=0x100000, k=0x200000, v=0x300000, qw=0x400000, kw=0x410000, qo=0x500000, T=3, B=2, H=4, Hkv=2, D=64,
           qs=256, ks=128, vs=128, eps=1e-6, rotate=1, center=3, dtype=1, **cache):
    c = f8_args(**cache) if cache.pop("null", 0) == 0 else None
    return name(lib.dilated_attn_cache_append_f8(q, k, v, qw, kw, qo, c, T, B, H, Hkv, D, qs, ks, vs, eps, rotate, center,
                                                 10000.0, 0.4, 512.0, dtype, None))


@pytest.mark.parametrize("change, code", [
    (dict(T=0, q=None, qo=None, k=None, v=None, qw=None), "DA_OK"), (dict(k=None), "DA_EINVAL"), (dict(v=None), "DA_EINVAL"),
    (dict(qo=None), "DA_EINVAL"), (dict(k_scale=None), "DA_EINVAL"), (dict(v_scale=None), "DA_EINVAL"),
    (dict(T=1 << 30, B=1 << 30), "DA_EINVAL"), (dict(k=0x200008), "DA_EALIGN"), (dict(ks=130), "DA_EALIGN"),
    (dict(D=48, qs=192), "DA_EUNSUPPORTED"), (dict(dtype=2), "DA_EUNSUPPORTED"), (dict(rotate=2), "DA_EINVAL"),
    (dict(center=-1), "DA_EINVAL"), (dict(eps=0.0), "DA_EINVAL"), (dict(k_scale=0x1000000), "DA_EINVAL"),
    (dict(v_scale=0x5000010), "DA_EINVAL"), (dict(k_scale=0x200010), "DA_EINVAL"), (dict(page_size=24), "DA_EINVAL"),
    (dict(num_pages=0), "DA_EINVAL"), (dict(k=0x2000000), "DA_EINVAL"), (dict(seq_lens=0x3100002), "DA_EALIGN"),
], ids=str)
def test_append_refuses(lib, change, code):
    assert append(lib, **change) == code
    if code == "DA_OK":
        from paper_2307_02486_amd import _lib
        assert name(lib.dilated_attn_cache_append_f8(*[None] * 6, None, 0, 1, 1, 1, 64, 64, 64, 64, 1e-6, 0, 0, 1e4, 0.4,
                                                     512.0, 1, None)) == "DA_EINVAL"


def attend(lib, q=0x100000, out=0x200000, lse=0x300000, T=3, B=2, H=4, Hkv=2, D=64, qs=256, max_new=3, dtype=1, scale=0.0,
           ws=0x8000000, ws_bytes=1 << 24, patterns=((64, 1),), **cache):
    from paper_2307_02486_amd import _lib
    arr, n = _lib.pattern_array(patterns)
    return name(lib.dilated_attn_paged_fwd_f8(q, f8_args(**cache), out, lse, T, B, H, Hkv, D, qs, max_new, arr, n, dtype,
                                              scale, ws, ws_bytes, None))


@pytest.mark.parametrize("change, code", [
    (dict(T=0, q=0, out=0, lse=0, ws=0, ws_bytes=0), "DA_OK"), (dict(k_scale=None), "DA_EINVAL"),
    (dict(v_scale=None), "DA_EINVAL"), (dict(q=0), "DA_EINVAL"), (dict(out=0x200004), "DA_EALIGN"),
    (dict(ws_bytes=64), "DA_EWORKSPACE"), (dict(out=0x5000000), "DA_EINVAL"), (dict(ws=0x5100000), "DA_EINVAL"),
    (dict(lse=0x5000004), "DA_EINVAL"), (dict(H=3), "DA_EINVAL"), (dict(dtype=2), "DA_EUNSUPPORTED"),
    (dict(scale=float("nan")), "DA_EINVAL"), (dict(v=None), "DA_EINVAL"),
], ids=str)
def test_paged_fwd_refuses(lib, change, code):
    assert attend(lib, **change) == code


def weigh(lib, q=0x100000, lse=0x300000, weights=0x310000, T=3, B=2, H=4, Hkv=2, D=64, qs=256, dtype=1, scale=0.0,
          ws=0x8000000, ws_bytes=1 << 24, patterns=((64, 1),), max_new=0, **cache):
    from paper_2307_02486_amd import _lib
    arr, n = _lib.pattern_array(patterns)
    return name(lib.dilated_attn_page_weights(q, lse, f8_args(**cache), weights, T, B, H, Hkv, D, qs, max_new, arr, n, dtype,
                                              scale, ws, ws_bytes, None))


@pytest.mark.parametrize("change, code", [
    (dict(T=0, q=0, lse=0, weights=0, ws=0, ws_bytes=0, v=None, v_scale=None), "DA_OK"), (dict(k_scale=None), "DA_EINVAL"),
    (dict(q=0), "DA_EINVAL"), (dict(lse=0), "DA_EINVAL"), (dict(weights=0), "DA_EINVAL"), (dict(ws=0), "DA_EINVAL"),
    (dict(lse=0x300002), "DA_EALIGN"), (dict(weights=0x310001), "DA_EALIGN"), (dict(ws=0x8000008), "DA_EALIGN"),
    (dict(ws_bytes=16), "DA_EWORKSPACE"), (dict(weights=0x5000000), "DA_EINVAL"), (dict(ws=0x1000000), "DA_EINVAL"),
    (dict(weights=0x300004), "DA_EINVAL"), (dict(weights=0x8000010), "DA_EINVAL"), (dict(D=96), "DA_EUNSUPPORTED"),
    (dict(scale=-1.0), "DA_EINVAL"), (dict(k=None), "DA_EINVAL"), (dict(max_new=-1), "DA_EINVAL"),
], ids=str)
def test_page_weights_refuses(lib, change, code):
    assert weigh(lib, **change) == code


@pytest.mark.parametrize("change, code", [
    (dict(weights=None), "DA_EINVAL"), (dict(table=None), "DA_EINVAL"), (dict(lens=None), "DA_EINVAL"),
    (dict(out=None), "DA_EINVAL"), (dict(freed=None), "DA_EINVAL"), (dict(count=None), "DA_EINVAL"), (dict(B=0), "DA_EINVAL"),
    (dict(num_pages=0), "DA_EINVAL"), (dict(page=10), "DA_EINVAL"), (dict(page=1 << 17), "DA_EINVAL"),
    (dict(max_pages=0), "DA_EINVAL"), (dict(max_pages=1 << 28), "DA_EINVAL"), (dict(keep=-1), "DA_EINVAL"),
    (dict(first=-1), "DA_EINVAL"), (dict(last=-1), "DA_EINVAL"), (dict(weights=0x1002), "DA_EALIGN"),
    (dict(freed=0x20004), "DA_EINVAL"), (dict(out=0x20004), "DA_EINVAL"), (dict(out=0x1004), "DA_EINVAL"),
    (dict(count=0x30000), "DA_EINVAL"), (dict(count=0x40004), "DA_EINVAL"),
], ids=str)
def test_evict_refuses(lib, change, code):
    a = dict(weights=0x1000, table=0x20000, lens=0x30000, out=0x40000, freed=0x50000, count=0x60000, B=2, num_pages=10,
             page=16, max_pages=4, keep=1, first=0, last=0)
    a.update(change)
    assert name(lib.dilated_attn_evict_pages(*a.values(), None)) == code


# -- the binding --------------------------------------------------------------------
def test_binding_refuses_host_tensors():
    from paper_2307_02486_amd import cache_append, cache_scale_shape, evict_pages, page_weights, paged_attn
    z = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c = z(4, 2, 32, 64, d=torch.uint8).view(F8)
    assert cache_scale_shape(c) == (4, 2, 2) and cache_scale_shape(c[:, :, :8]) == (4, 2, 1)
    s = z(4, 2, 2, d=torch.uint8).view(E8)
    with pytest.raises(RuntimeError, match="GPU only"):
        cache_append(None, z(3, 2, 64), z(3, 2, 64), c, c, i(1, 4), i(1), i(2), k_scale=s, v_scale=s)
    with pytest.raises(RuntimeError, match="GPU only"):
        paged_attn(z(3, 4, 64), c, c, i(1, 4), i(1), i(2), [(8, 1)], k_scale=s, v_scale=s)
    with pytest.raises(RuntimeError, match="GPU only"):
        page_weights(z(3, 4, 64), z(4, 3, d=torch.float32), c, s, i(1, 4), i(1), i(2), [(8, 1)], z(4, d=torch.float32))
    with pytest.raises(RuntimeError, match="GPU only"):
        evict_pages(z(4, d=torch.float32), i(1, 4), i(1), 16, 2)


def test_calls_run_on_the_tensors_device(monkeypatch):
    """Stream 0 is the current device's: a call for another device makes that current."""
    from paper_2307_02486_amd import ops
    now, seen = [0], []

    class On:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.was, now[0] = now[0], self.dev

        def __exit__(self, *_):
            now[0] = self.was

    monkeypatch.setattr(ops.torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(ops.torch.cuda, "device", On)
    for dev in (0, 1):
        assert ops._call_on(dev, lambda *x: seen.append((now[0], x)) or 7, "a", 2) == 7
    assert seen == [(0, ("a", 2)), (1, ("a", 2))] and now == [0]


def test_scales_are_checked():
    from paper_2307_02486_amd.ops import _check_scale
    c = torch.zeros((4, 2, 32, 64), dtype=torch.uint8).view(F8)
    good = torch.zeros((4, 2, 2), dtype=torch.uint8)
    _check_scale("k_scale", good.view(E8), c)
    for bad in (None, good, good.view(E8)[:, :, :1], good.view(E8)[:2], good.view(E8).transpose(1, 2)):
        with pytest.raises(ValueError, match="k_scale"):
            _check_scale("k_scale", bad, c)


# -- the cache's pages ----------------------------------------------------------------
def test_a_cache_in_8_bits_has_scales():
    from paper_2307_02486_amd.serving import PagedCache
    cache = PagedCache(6, 32, 4, 2, 64, layers=2, device="cpu", dtype=F8, weigh=True)
    assert [s.shape for s in cache.k_scale + cache.v_scale] == [(6, 2, 2)] * 4 and cache.k_scale[0].dtype == E8
    assert cache.k[1].dtype == F8 and cache.weights.tolist() == [0.0] * 6
    wide = PagedCache(6, 32, 4, 2, 64, device="cpu")
    assert wide.k_scale is None and wide.weights is None
    with pytest.raises(ValueError, match="weigh"):
        PagedCache(6, 32, 4, 2, 64, device="cpu", weigh=True)
    with pytest.raises(ValueError, match="weigh"):
        wide.evict(1)


def test_pages_that_are_gone_stay_gone(monkeypatch):
    """Evicted pages go back to the pool and are -1 in later tables; the sequence
    grows on behind them, is taken back and released around them."""
    from paper_2307_02486_amd import serving
    cache = serving.PagedCache(10, 4, 8, 1, 64, device="cpu", dtype=F8, weigh=True)
    cache.extend(["a", "b"], [22, 5])
    a = list(cache._pages["a"])
    cache.weights[:] = torch.arange(10.0)
    cache.weights[a[3]] = -1.0

    def evict(weights, table, lens, page, keep, first, last):
        got = evict_ref(weights.numpy(), table.numpy(), lens.numpy(), page, keep, first, last)
        return tuple(torch.from_numpy(x) for x in got)

    monkeypatch.setattr(serving, "evict_pages", evict)
    with pytest.raises(ValueError):
        cache.evict(-1)
    with pytest.raises(ValueError, match="last"):
        cache.evict(2, last=0)  # the next tokens need it
    with pytest.raises(ValueError):
        cache.evict(2, ["a", "x"])
    with pytest.raises(ValueError):
        cache.evict(2, ["a", "a"])
    last = cache.extend(["a"], [1])
    assert cache.evict(4, ["a"]) == 2
    gone = [j for j, p in enumerate(cache._pages["a"]) if p < 0]
    assert 3 in gone and len(gone) == 2 and set(a[j] for j in gone) <= set(cache._free)
    with pytest.raises(ValueError):
        cache.retract(last)  # the batch names pages that went
    batch = cache.extend(["a", "b"], [3, 0])
    row = batch.block_table[0].tolist()
    assert [row[j] for j in gone] == [-1, -1] and row[:7].count(-1) == 2 and row[7] == -1 and int(batch.seq_lens[0]) == 26
    taken = row[6]
    assert cache.weights[taken] == 0.0
    cache.retract(batch)
    assert cache.length("a") == 23 and taken in cache._free
    assert cache.evict(4) == 0
    cache.release("a")
    cache.release("b")
    assert sorted(cache._free) == list(range(10))
    assert cache.evict(1) == 0
