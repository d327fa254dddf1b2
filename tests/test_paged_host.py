"""Host side of the head norms and of the paged cache: refusals of the C ABI and
of the binding, the paged plan's workspace, the cache's page keeping, and the
oracles against the ones that are there.  No GPU."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle.layer_ref import XPosConfig, xpos_ref
from oracle.paged_ref import heads_ref, paged_attention_ref


@pytest.fixture(scope="module")
def lib():
    from paper_2307_02486_amd import _lib
    return _lib.load()


def name(rc):
    from paper_2307_02486_amd import _lib
    return _lib.ERRORS[rc]


def test_exports_the_declared_symbols(lib):
    for n in ("dilated_attn_qk_norm_xpos", "dilated_attn_qk_norm_xpos_bwd_workspace", "dilated_attn_qk_norm_xpos_bwd",
              "dilated_attn_cache_append", "dilated_attn_paged_workspace", "dilated_attn_paged_fwd"):
        assert hasattr(lib, n)


# -- oracles -----------------------------------------------------------------
@pytest.mark.parametrize("patterns", [[(8, 1), (16, 3)], [(5, 2), (40, 1), (1 << 40, 7)], [(1, 1)]], ids=str)
def test_paged_oracle_is_the_operator_on_the_sequence(patterns):
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(1, 37, 4, 8)) for _ in range(3))
    want, want_lse = oracle.dilated_attention_ref(q, k, v, [(min(w, 37), min(r, w, 37)) for w, r in patterns], True)
    out, lse = paged_attention_ref(q[0, 20:], k[0], v[0], 20, patterns)
    assert np.allclose(out, want[0, 20:], atol=1e-12)
    assert np.allclose(lse.T, want_lse[0, :, 20:], atol=1e-12)


def test_heads_oracle_without_norm_is_xpos():
    x = np.random.default_rng(2).normal(size=(1, 50, 2, 16))
    cfg = XPosConfig(center=11)
    for sign in (1, -1):
        assert np.allclose(heads_ref(x, None, np.arange(50), sign, 11), xpos_ref(x, sign, cfg), atol=1e-12)


# -- the paged plan ----------------------------------------------------------
def need(T=8, B=2, H=4, Hkv=2, D=64, num_pages=10, page=16, max_pages=4, patterns=((64, 1),), max_new=None, dtype=torch.bfloat16):
    from paper_2307_02486_amd import paged_workspace_bytes
    return paged_workspace_bytes(T, B, H, Hkv, D, num_pages, page, max_pages, patterns, max_new, dtype)


def test_workspace_holds_every_partial_row():
    """A single token needs a float32 row and a float of each of its slots, a
    tile's row an fp16 row and its record of each pattern."""
    assert need(T=1, B=1) >= 4 * (64 * 4 + 4)
    assert need(T=200, B=2) >= 200 * 4 * (64 * 2 + 8)
    assert need(T=200, B=2, patterns=((64, 1), (64, 2))) >= 2 * 200 * 4 * (64 * 2 + 8)
    assert need(T=0) >= 0
    assert need(T=200, B=200, max_new=1) < need(T=200, B=200)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(B=0), dict(H=0), dict(H=5), dict(Hkv=0), dict(H=1 << 16, Hkv=1), dict(num_pages=0), dict(page=12),
    dict(page=0), dict(page=1 << 17), dict(max_pages=0), dict(max_pages=1 << 28), dict(num_pages=1 << 31), dict(max_new=-1),
    dict(patterns=()), dict(patterns=((4, 8),)), dict(patterns=((0, 1),)), dict(patterns=((8, 1),) * 17),
    dict(T=1 << 30, H=8, Hkv=8, B=1 << 20),
], ids=str)
def test_plan_refuses(change):
    from paper_2307_02486_amd import DilatedAttnError
    with pytest.raises(DilatedAttnError) as e:
        need(**change)
    assert e.value.name == "DA_EINVAL"


def test_plan_refuses_types_and_sizes():
    from paper_2307_02486_amd import DilatedAttnError
    for change in (dict(D=40), dict(D=256)):
        with pytest.raises(DilatedAttnError) as e:
            need(**change)
        assert e.value.name == "DA_EUNSUPPORTED"
    with pytest.raises(TypeError):
        need(dtype=torch.float16)


# -- the C ABI, with pointers that are never followed --------------------------
def cache_args(**change):
    from paper_2307_02486_amd import _lib
    c = dict(k=0x1000000, v=0x2000000, block_table=0x3000000, seq_lens=0x3100000, q_start=0x3200000, num_pages=10,
             page_size=16, max_pages=4)
    c.update(change)
    return _lib.PagedCacheArgs(*c.values())


def paged_fwd(lib, q=0x100000, out=0x200000, lse=0x300000, T=3, B=2, H=4, Hkv=2, D=64, qs=256, max_new=3, dtype=1,
              scale=0.0, ws=0x4000000, ws_bytes=1 << 24, patterns=((64, 1),), cache=None):
    from paper_2307_02486_amd import _lib
    arr, n = _lib.pattern_array(patterns)
    c = cache_args() if cache is None else cache
    return name(lib.dilated_attn_paged_fwd(q, c, out, lse, T, B, H, Hkv, D, qs, max_new, arr, n, dtype, scale, ws, ws_bytes, None))


@pytest.mark.parametrize("change, code", [
    (dict(q=0), "DA_EINVAL"), (dict(out=0), "DA_EINVAL"), (dict(lse=0), "DA_EINVAL"), (dict(ws=0), "DA_EINVAL"),
    (dict(q=0x100008), "DA_EALIGN"), (dict(out=0x200004), "DA_EALIGN"), (dict(lse=0x300002), "DA_EALIGN"),
    (dict(ws=0x4000008), "DA_EALIGN"), (dict(ws_bytes=64), "DA_EWORKSPACE"), (dict(qs=252), "DA_EINVAL"),
    (dict(qs=260), "DA_EALIGN"), (dict(qs=1 << 33), "DA_EINVAL"), (dict(H=3), "DA_EINVAL"), (dict(D=48), "DA_EUNSUPPORTED"),
    (dict(dtype=2), "DA_EUNSUPPORTED"), (dict(scale=-1.0), "DA_EINVAL"), (dict(scale=float("inf")), "DA_EINVAL"),
    (dict(out=0x1000100), "DA_EINVAL"), (dict(out=0x100000), "DA_EINVAL"), (dict(lse=0x200000), "DA_EINVAL"),
    (dict(ws=0x2000000), "DA_EINVAL"), (dict(ws=0x3000000), "DA_EINVAL"), (dict(T=-1), "DA_EINVAL"),
    (dict(max_new=-2), "DA_EINVAL"), (dict(patterns=((2, 4),)), "DA_EINVAL"),
    (dict(T=0, q=0, out=0, lse=0, ws=0, ws_bytes=0), "DA_OK"),
], ids=str)
def test_paged_fwd_refuses(lib, change, code):
    assert paged_fwd(lib, **change) == code


@pytest.mark.parametrize("change, code", [
    (dict(k=0), "DA_EINVAL"), (dict(v=0), "DA_EINVAL"), (dict(block_table=0), "DA_EINVAL"), (dict(seq_lens=0), "DA_EINVAL"),
    (dict(q_start=0), "DA_EINVAL"), (dict(num_pages=0), "DA_EINVAL"), (dict(page_size=24), "DA_EINVAL"),
    (dict(max_pages=0), "DA_EINVAL"), (dict(max_pages=1 << 27), "DA_EINVAL"), (dict(k=0x1000008), "DA_EALIGN"),
    (dict(q_start=0x3200002), "DA_EALIGN"),
], ids=str)
def test_both_paged_calls_refuse_the_cache(lib, change, code):
    assert paged_fwd(lib, cache=cache_args(**change)) == code
    assert append(lib, cache=cache_args(**change)) == code


def append(lib, q=0x100000, k=0x200000, v=0x300000, qw=0, kw=0, qo=0x400000, T=3, B=2, H=4, Hkv=2, D=64, qs=256, ks=128,
           vs=128, eps=1e-6, rotate=1, center=10, base=1e4, gamma=0.4, scale_base=512.0, dtype=1, cache=None):
    c = cache_args() if cache is None else cache
    return name(lib.dilated_attn_cache_append(q, k, v, qw, kw, qo, c, T, B, H, Hkv, D, qs, ks, vs, eps, rotate, center, base,
                                              gamma, scale_base, dtype, None))


@pytest.mark.parametrize("change, code", [
    (dict(k=0), "DA_EINVAL"), (dict(v=0), "DA_EINVAL"), (dict(qo=0), "DA_EINVAL"), (dict(q=0), "DA_EINVAL"),
    (dict(k=0x200008), "DA_EALIGN"), (dict(kw=0x500008), "DA_EALIGN"), (dict(ks=120), "DA_EINVAL"), (dict(vs=132), "DA_EALIGN"),
    (dict(D=96), "DA_EUNSUPPORTED"), (dict(dtype=3), "DA_EUNSUPPORTED"), (dict(T=1 << 31), "DA_EINVAL"), (dict(B=0), "DA_EINVAL"),
    (dict(rotate=2), "DA_EINVAL"), (dict(center=64), "DA_EINVAL"), (dict(center=-1), "DA_EINVAL"), (dict(base=1.0), "DA_EINVAL"),
    (dict(gamma=0.0), "DA_EINVAL"), (dict(scale_base=0.5), "DA_EINVAL"), (dict(kw=0x500000, eps=0.0), "DA_EINVAL"),
    (dict(kw=0x500000, eps=1e-40), "DA_EINVAL"), (dict(qw=0x500000, eps=float("nan")), "DA_EINVAL"),
    (dict(qo=0x1000000), "DA_EINVAL"), (dict(qo=0x200000), "DA_EINVAL"), (dict(k=0x1000200), "DA_EINVAL"),
    (dict(T=0, k=0, v=0, q=0, qo=0), "DA_OK"),
], ids=str)
def test_append_refuses(lib, change, code):
    assert append(lib, **change) == code


def test_append_looks_at_what_it_uses_only(lib):
    nan = float("nan")
    assert append(lib, T=0, eps=nan) == "DA_OK"  # no weights
    assert append(lib, T=0, rotate=0, center=-5, base=nan, gamma=nan, scale_base=nan) == "DA_OK"


def norm(lib, bwd=False, q=0x100000, k=0x200000, qw=0x300000, kw=0x310000, qo=0x400000, ko=0x500000, B=1, N=4, H=4, Hkv=2,
         D=64, qs=256, ks=128, eps=1e-6, center=2, base=1e4, gamma=0.4, scale_base=512.0, dtype=1, ws=0xA00000, ws_bytes=1 << 20,
         dq=0x600000, dk=0x700000, dqw=0x800000, dkw=0x900000):
    tail = (B, N, H, Hkv, D, qs, ks, eps, center, base, gamma, scale_base, dtype)
    if bwd:
        return name(lib.dilated_attn_qk_norm_xpos_bwd(qo, ko, q, k, qw, kw, dq, dk, dqw, dkw, *tail, ws, ws_bytes, None))
    return name(lib.dilated_attn_qk_norm_xpos(q, k, qw, kw, qo, ko, *tail, None))


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("change, code", [
    (dict(q=0), "DA_EINVAL"), (dict(kw=0), "DA_EINVAL"), (dict(ko=0), "DA_EINVAL"), (dict(k=0x200004), "DA_EALIGN"),
    (dict(qs=248), "DA_EINVAL"), (dict(qs=257), "DA_EALIGN"), (dict(B=0), "DA_EINVAL"), (dict(N=0), "DA_EINVAL"),
    (dict(N=1 << 31), "DA_EINVAL"), (dict(H=0), "DA_EINVAL"), (dict(Hkv=1 << 16, ks=1 << 22), "DA_EINVAL"), (dict(D=80), "DA_EUNSUPPORTED"),
    (dict(dtype=7), "DA_EUNSUPPORTED"), (dict(eps=0.0), "DA_EINVAL"), (dict(eps=float("inf")), "DA_EINVAL"),
    (dict(center=4), "DA_EINVAL"), (dict(base=0.5), "DA_EINVAL"), (dict(scale_base=0.01), "DA_EINVAL"),
], ids=str)
def test_norm_refuses(lib, bwd, change, code):
    assert norm(lib, bwd, **change) == code


@pytest.mark.parametrize("change, code", [
    (dict(dq=0), "DA_EINVAL"), (dict(dkw=0), "DA_EINVAL"), (dict(ws=0), "DA_EINVAL"), (dict(ws=0xA00004), "DA_EALIGN"),
    (dict(ws_bytes=16), "DA_EWORKSPACE"), (dict(dq=0x100000), "DA_EINVAL"), (dict(dk=0x600000), "DA_EINVAL"),
    (dict(dqw=0x300000), "DA_EINVAL"), (dict(ws=0x700000), "DA_EINVAL"),
], ids=str)
def test_norm_bwd_refuses(lib, change, code):
    assert norm(lib, True, **change) == code


def test_norm_forward_refuses_overlap(lib):
    assert norm(lib, qo=0x100000) == "DA_EINVAL"
    assert norm(lib, ko=0x400000) == "DA_EINVAL"


# -- the binding ---------------------------------------------------------------
def test_token_stride():
    from paper_2307_02486_amd.ops import _token_stride
    x = torch.zeros(3, 5, 12, 8, dtype=torch.bfloat16)
    d = (torch.bfloat16, x.device)
    assert _token_stride("x", x, 2, *d) == 96
    assert _token_stride("x", x[:, :, 2:6], 2, *d) == 96
    assert _token_stride("x", x[1, :, :4], 1, *d) == 96
    assert _token_stride("x", x[:, ::5], 2, *d) == 480      # one token of each sequence
    assert _token_stride("x", x[:1, :1, :3], 2, *d) == 24
    for bad in (x[:, ::2], x[:, :4], x.transpose(2, 3), x[..., ::2], x[:, :, ::2]):
        with pytest.raises(ValueError):
            _token_stride("x", bad, 2, *d)


def test_binding_refuses_what_is_not_on_the_gpu():
    import paper_2307_02486_amd as da
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    w, i = torch.ones(64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(RuntimeError):
        da.qk_norm_xpos(q, q, w, w)
    with pytest.raises(RuntimeError):
        da.qk_norm_xpos_bwd(q, q, q, q, w, w)
    kc = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    for _ in range(2):  # what is refused is not remembered
        with pytest.raises(RuntimeError):
            da.cache_append(q[0], q[0], q[0], kc, kc, i[None], i[:1], i)
        with pytest.raises(RuntimeError):
            da.paged_attn(q[0], kc, kc, i[None], i[:1], i, [(8, 1)])


# -- the cache's pages -----------------------------------------------------------
def test_page_keeping():
    from paper_2307_02486_amd.serving import PagedCache
    cache = PagedCache(6, 4, 4, 2, 32, layers=2, device="cpu")
    assert len(cache.k) == len(cache.v) == 2 and cache.k[0].shape == (6, 2, 4, 32) and cache.center == 8
    b = cache.extend(["a", "b"], [5, 1])
    assert b.seq_lens.tolist() == [5, 1] and b.q_start.tolist() == [0, 5, 6] and b.max_new == 5
    used = b.block_table[0, :2].tolist() + b.block_table[1, :1].tolist()
    assert len(set(used)) == 3
    b = cache.extend(["b", "a"], [3, 3])  # b fills its page, a its two
    assert b.seq_lens.tolist() == [4, 8] and b.block_table[1, :2].tolist() == used[:2]
    with pytest.raises(ValueError):
        cache.extend(["a"], [9])          # beyond the table
    with pytest.raises(RuntimeError):
        cache.extend(["c"], [16])         # beyond the pool
    assert cache.length("c") == 0 and cache.length("a") == 8  # a refusal changes nothing
    cache.release("a")
    assert cache.length("a") == 0
    b = cache.extend(["c"], [16])
    assert sorted(b.block_table[0].tolist() + [used[2]]) == sorted(set(b.block_table[0].tolist() + [used[2]]))
    for bad in (lambda: cache.extend(["x", "x"], [1, 1]), lambda: cache.extend(["x"], [-1]), lambda: cache.extend([], []),
                lambda: PagedCache(4, 6, 2, 1, 32, device="cpu"), lambda: PagedCache(0, 4, 2, 1, 32, device="cpu")):
        with pytest.raises(ValueError):
            bad()


def test_layer_refuses_head_norms_without_rotation():
    from paper_2307_02486_amd.layer import LongNetAttention
    with pytest.raises(ValueError):
        LongNetAttention(64, 2, [(8, 1)], use_xpos=False, qk_norm=True, device="cpu")
    layer = LongNetAttention(64, 2, [(8, 1)], qk_norm=True, device="cpu")
    assert set(layer.float64_params()) >= {"q_norm", "k_norm"} and layer.q_norm.shape == (32,)
    assert "q_norm" not in LongNetAttention(64, 2, [(8, 1)], device="cpu").state_dict()
    assert ctypes.sizeof(ctypes.c_void_p) == 8
