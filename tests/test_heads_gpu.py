"""The head norms with xPos (both directions) and the cache append against float64.

Bars, per element unless said otherwise (u = 2^-8 for bf16 outputs, 2^-24 for
float32: half the spacing of 8 and of 24 significant bits, the rounding of the
output itself):
  * forward: |y - ref| <= u |ref| + 4e-6 |ref pair|: float32 norm (a sum of at
    most 128 squares, one reciprocal root), series for sine and cosine (3e-8),
    scale (two roundings of an exponent below 1 and an exp2), six products.
  * dx: |dx - ref| <= u |ref| + 2e-5 max over the row of (|dn w| + |xhat m|) rstd:
    the two terms cancel, their sum's roundings do not.
  * dw: |dw - ref| <= u |ref| + 1e-5 sum of |terms|: float32 sums of up to some
    thousand terms a lane, then pairwise.
  * gradients by differences (float64 forward, step 1e-6): 1e-6 relative: the
    formula of the reference itself.
"""
import numpy as np
import pytest
import torch

import workloads
from oracle.paged_ref import heads_bwd_ref, heads_ref
from tests.gpu_util import note, require_gpu, to64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def unit(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


def check(y, ref, dtype, tag, slack=4e-6, size=None):
    y = to64(y)
    if size is None:
        pair = np.hypot(ref[..., 0::2], ref[..., 1::2])
        size = np.repeat(pair, 2, axis=-1)
    bad = np.abs(y - ref) > unit(dtype) * 1.001 * np.abs(ref) + slack * size + 1e-37
    assert not bad.any(), f"{tag}: {bad.sum()} of {bad.size}, worst {np.abs(y - ref).max()}"


def draw(shape, dtype, seed, tid, sigma=1.0):
    return workloads.make_random(shape, dtype, sigma, seed, "cuda", tid)


CASES = [
    # (B, N, H, Hkv, D, dtype, sliced, center)
    (1, 1, 1, 1, 64, BF, False, 0),
    (2, 37, 12, 12, 64, BF, False, None),
    (1, 300, 5, 3, 128, BF, True, 7),
    (3, 129, 17, 2, 32, BF, True, None),
    (1, 32768, 3, 1, 64, BF, False, None),      # angles of 32767 radians, scales of 2^+-58
    (2, 65, 6, 2, 32, F32, True, None),
    (1, 32768, 1, 2, 64, F32, False, None),
    (1, 9, 40, 33, 128, F32, False, 8),         # more heads than a wave holds at once
]


def qk_of(case):
    B, N, H, Hkv, D, dtype, sliced, _ = case
    if sliced:
        x = draw((B, N, H + 2 * Hkv, D), dtype, 41 + N, 0)
        return x[:, :, :H], x[:, :, H: H + Hkv]
    return draw((B, N, H, D), dtype, 41 + N, 0), draw((B, N, Hkv, D), dtype, 41 + N, 1)


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c)[:44])
def test_norm_forward_and_backward(case):
    from paper_2307_02486_amd import qk_norm_xpos, qk_norm_xpos_bwd
    B, N, H, Hkv, D, dtype, _, center = case
    note(f"[heads] {case}")
    q, k = qk_of(case)
    qw, kw = (draw((D,), dtype, 43 + N, t, 0.3) + 1 for t in (0, 1))
    qo, ko = qk_norm_xpos(q, k, qw, kw, center=center)
    dqo, dko = draw((B, N, H, D), dtype, 47 + N, 0), draw((B, N, Hkv, D), dtype, 47 + N, 1)
    first = qk_norm_xpos_bwd(dqo, dko, q, k, qw, kw, center=center)
    again = qk_norm_xpos_bwd(dqo, dko, q, k, qw, kw, center=center)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    dq, dk, dqw, dkw = first
    c = N // 2 if center is None else center
    for x, w, y, dy, dx, dw, sign in ((q, qw, qo, dqo, dq, dqw, 1), (k, kw, ko, dko, dk, dkw, -1)):
        assert y.is_contiguous() and dx.is_contiguous() and y.shape == x.shape == dx.shape
        x64, w64, dy64, pos = to64(x), to64(w), to64(dy), np.arange(N)
        check(y, heads_ref(x64, w64, pos, sign, c), dtype, "forward")
        rx, rw = heads_bwd_ref(dy64, x64, w64, pos, sign, c)
        rms = np.sqrt((x64 * x64).mean(-1, keepdims=True) + 1e-6)
        xhat = x64 / rms
        one = heads_ref(dy64, None, -pos, 1, 0, scale_base=1e30)  # the transposed rotation alone
        zeta = (2 * np.arange(D // 2) / D + 0.4) / 1.4
        one *= np.repeat(zeta ** (sign * (pos[:, None, None] - c) / 512.0), 2, axis=-1)
        g = np.abs(one * w64)
        size = ((g + np.abs(xhat) * (g * np.abs(xhat)).mean(-1, keepdims=True)) / rms).max(-1, keepdims=True)
        check(dx, rx, dtype, "dx", 2e-5, size)
        check(dw, rw, dtype, "dw", 1e-5, np.abs(one * xhat).reshape(-1, D).sum(0))


def test_reference_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(5)
    x, w, dy = rng.normal(size=(3, 2, 32)), rng.normal(size=32) + 1, rng.normal(size=(3, 2, 32))
    pos = np.array([0, 900, 2011])
    dx, dw = heads_bwd_ref(dy, x, w, pos, -1, 100)
    f = lambda x, w: (heads_ref(x, w, pos, -1, 100) * dy).sum()  # noqa: E731
    for _ in range(20):
        ex, ew = rng.normal(size=x.shape), rng.normal(size=w.shape)
        for d, along in ((ex, ((dx * ex).sum())), (None, (dw * ew).sum())):
            h = 1e-6
            num = (f(x + h * d, w) - f(x - h * d, w)) / (2 * h) if d is not None else (f(x, w + h * ew) - f(x, w - h * ew)) / (2 * h)
            assert abs(num - along) <= 1e-6 * (1 + abs(along) + np.abs(dy).sum())


def test_kernel_gradient_against_differences_of_the_kernel():
    """Float32: the loss sum(y dy) along random directions; steps of 1e-2 of smooth
    functions of size 1 leave 1e-3 relative, float32 sums less."""
    from paper_2307_02486_amd import qk_norm_xpos, qk_norm_xpos_bwd
    note("[heads] differences")
    q, k = draw((1, 6, 4, 32), F32, 61, 0), draw((1, 6, 2, 32), F32, 61, 1)
    qw, kw = draw((32,), F32, 62, 0, 0.2) + 1, draw((32,), F32, 62, 1, 0.2) + 1
    dqo, dko = draw((1, 6, 4, 32), F32, 63, 0), draw((1, 6, 2, 32), F32, 63, 1)
    grads = qk_norm_xpos_bwd(dqo, dko, q, k, qw, kw)

    def loss(args):
        y = qk_norm_xpos(*args)
        return (y[0].double() * dqo).sum() + (y[1].double() * dko).sum()

    for i in range(4):
        args = [q, k, qw, kw]
        for seed in range(3):
            e = draw(args[i].shape, F32, 70 + seed, i)
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + 1e-2 * e, args[i] - 1e-2 * e
            num = float((loss(up) - loss(down)) / 2e-2)
            along = float((grads[i].double() * e).sum())
            scale = float((grads[i].double() * e).abs().sum())
            assert abs(num - along) <= 1e-3 * scale, (i, seed, num, along)


def test_zero_rows_and_large_values():
    """A head of zeros norms to zeros (eps keeps the root finite); bf16 heads
    around 1e18, whose squares stay finite in float32, norm like others."""
    from paper_2307_02486_amd import qk_norm_xpos, qk_norm_xpos_bwd
    note("[heads] extremes")
    q, k = draw((1, 4, 3, 64), BF, 81, 0), draw((1, 4, 3, 64), BF, 81, 1)
    q[0, 1, 2] = 0
    k = (k.float() * 1e18).to(BF)
    w = torch.ones(64, dtype=BF, device="cuda")
    qo, ko = qk_norm_xpos(q, k, w, w)
    assert bool((qo[0, 1, 2] == 0).all())
    check(ko, heads_ref(to64(k), np.ones(64), np.arange(4), -1, 2), BF, "large")
    grads = qk_norm_xpos_bwd(torch.ones_like(qo), torch.ones_like(ko), q, k, w, w)
    assert all(bool(torch.isfinite(g).all()) for g in grads)


APPENDS = [
    # (new tokens, cached before, H, Hkv, D, page, dtype, norm, rotate, sliced, with q)
    ([1], [0], 4, 4, 64, 16, BF, False, True, False, True),
    ([1, 1, 1, 1, 1], [0, 15, 16, 200, 63], 12, 12, 64, 16, BF, True, True, True, True),
    ([70, 0, 3, 129], [5, 9, 0, 63], 8, 2, 128, 64, BF, True, True, True, True),
    ([33, 1], [0, 31], 6, 3, 32, 1, BF, False, False, False, True),
    ([17, 40], [3, 0], 5, 5, 64, 8, F32, True, True, True, True),
    ([20], [100], 3, 3, 128, 256, F32, False, True, False, False),
    ([1] * 70, list(range(70)), 2, 1, 64, 32, BF, False, True, False, True),
]


def paged(new, before, page, extra_pages=3, seed=0):
    """Tables of randomly ordered pages, lengths and starts for sequences."""
    blocks = [-(-(n + c) // page) for n, c in zip(new, before)]
    order = np.random.default_rng(seed).permutation(sum(blocks) + extra_pages)
    table = np.full((len(new), max(max(blocks), 1) + 2), 2 ** 30, dtype=np.int32)  # entries past a sequence are not used
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at: at + n]
        at += n
    lens = np.array([n + c for n, c in zip(new, before)], dtype=np.int32)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    dev = [torch.from_numpy(x).cuda() for x in (table, lens, start)]
    return table, lens, start, dev, len(order)


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: str(c)[:50])
def test_append(case):
    from paper_2307_02486_amd import cache_append
    new, before, H, Hkv, D, page, dtype, norm, rotate, sliced, with_q = case
    note(f"[append] {case}")
    table, lens, start, dev, pages = paged(new, before, page)
    T = int(start[-1])
    x = draw((T, H + 2 * Hkv, D), dtype, 51, 0)
    q, k, v = x[:, :H], x[:, H: H + Hkv], x[:, H + Hkv:]
    if not sliced:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    qw = draw((D,), dtype, 52, 0, 0.2) + 1 if norm and with_q else None
    kw = draw((D,), dtype, 52, 1, 0.2) + 1 if norm else None
    kc, vc = draw((pages, Hkv, page, D), dtype, 53, 0), draw((pages, Hkv, page, D), dtype, 53, 1)
    k0, v0 = kc.clone(), vc.clone()
    center = table.shape[1] * page // 2
    qo = cache_append(q if with_q else None, k, v, kc, vc, *dev, q_weight=qw, k_weight=kw, rotate=rotate, center=center)
    torch.cuda.synchronize()
    assert (qo is None) == (not with_q)
    held = np.zeros((pages, page), dtype=bool)
    kk, vv = to64(kc), to64(vc)
    for b in range(len(new)):
        pos = np.arange(before[b], lens[b])
        rows = slice(start[b], start[b + 1])
        p, s = table[b, pos // page], pos % page
        held[p, s] = True
        assert np.array_equal(vv[p, :, s], to64(v[rows]))
        at = pos if rotate else np.zeros_like(pos)
        c = center if rotate else 0
        check(torch.from_numpy(kk[p, :, s]), heads_ref(to64(k[rows]), None if kw is None else to64(kw), at, -1, c),
              dtype, f"k of {b}")
        if with_q:
            check(qo[rows], heads_ref(to64(q[rows]), None if qw is None else to64(qw), at, 1, c), dtype, f"q of {b}")
    free = torch.from_numpy(~held).cuda()
    for cache, old in ((kc, k0), (vc, v0)):  # every other place of the pool keeps its bits
        assert torch.equal(cache.transpose(1, 2)[free], old.transpose(1, 2)[free])


def test_append_leaves_out_what_has_no_place():
    """Tokens of no sequence, positions below zero or beyond the table and pages
    outside the pool write nothing; queries of the first three are zeros."""
    from paper_2307_02486_amd import cache_append
    note("[append] no place")
    page, Hkv, D = 16, 2, 64
    kc, vc = draw((4, Hkv, page, D), BF, 91, 0), draw((4, Hkv, page, D), BF, 91, 1)
    k0, v0 = kc.clone(), vc.clone()
    # sequence 0: three tokens but a length of one; 1: past its two pages; 2: bad pages; then two tokens of none
    table = torch.tensor([[0, 1], [2, 3], [-1, 4]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([1, 34, 17], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 3, 7, 9], dtype=torch.int32, device="cuda")
    x = draw((11, 3 * Hkv, D), BF, 92, 0)
    qo = cache_append(x[:, :Hkv], x[:, Hkv: 2 * Hkv], x[:, 2 * Hkv:], kc, vc, table, lens, start, center=5)
    torch.cuda.synchronize()
    written = torch.zeros(4, page, dtype=torch.bool, device="cuda")
    written[0, 0] = written[3, 14] = written[3, 15] = True
    for cache, old in ((kc, k0), (vc, v0)):
        assert torch.equal(cache.transpose(1, 2)[~written], old.transpose(1, 2)[~written])
    assert torch.equal(vc[0, :, 0], x[2, 2 * Hkv:]) and torch.equal(vc[3, :, 15], x[4, 2 * Hkv:])
    gone = [0, 1, 5, 6, 9, 10]
    assert bool((qo[gone] == 0).all())
    assert bool((qo[[2, 3, 4, 7, 8]] != 0).any(-1).all())


def test_append_of_nothing():
    from paper_2307_02486_amd import cache_append
    kc = torch.zeros(1, 2, 16, 64, dtype=BF, device="cuda")
    x = torch.zeros(0, 2, 64, dtype=BF, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    qo = cache_append(x, x, x, kc, kc.clone(), torch.zeros(1, 1, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32))
    assert qo.shape == (0, 2, 64)
