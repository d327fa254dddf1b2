"""Performance cases of the operators around a dilated-attention layer that serves and trains with normed heads.

    norm_fwd   qk_norm_xpos: the RMS norm of each query and key head with the xPos rotation in the same pass
    norm_bwd   qk_norm_xpos_bwd: its gradients (queries, keys, both weights)
    append     cache_append: new keys and values into a paged cache, the keys (and queries) rotated on the way
    attn       paged_attn: dilated attention of each sequence's new tokens over its paged cache

A case is a dict of plain values.  `patterns` is a text "w:r,w:r,...".  The lengths of a batch follow from the
case alone (`_lengths`).  With `own` false `run` computes the operators in elementary torch operations in float32,
with `own` true it calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PAPER = "2048:1,4096:2,8192:4,16384:6,32768:12"  # the paper's five patterns (Sec. 4.1)
BASE, GAMMA, SCALE_BASE, EPS = 10000.0, 0.4, 512.0, 1e-6


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
def _norm(kind, B, N, H, Hkv, D, dtype="bf16", fused=False, name=None):
    c = {"kind": kind, "B": B, "N": N, "H": H, "Hkv": Hkv, "D": D, "dtype": dtype, "fused": fused}
    return dict(c, name=name) if name else c


def _append(B, H, Hkv, D, page, new, ctx_lo, ctx_hi, norm, dtype="bf16", fused=False, lengths=1, name=None):
    c = {"kind": "append", "B": B, "H": H, "Hkv": Hkv, "D": D, "page": page, "new": new, "ctx_lo": ctx_lo,
         "ctx_hi": ctx_hi, "norm": norm, "dtype": dtype, "fused": fused, "lengths": lengths}
    return dict(c, name=name) if name else c


def _attn(B, H, Hkv, D, page, new, ctx_lo, ctx_hi, patterns, dtype="bf16", lengths=1, name=None):
    c = {"kind": "attn", "B": B, "H": H, "Hkv": Hkv, "D": D, "page": page, "new": new, "ctx_lo": ctx_lo,
         "ctx_hi": ctx_hi, "patterns": patterns, "dtype": dtype, "lengths": lengths}
    return dict(c, name=name) if name else c


def listed():
    return [
        # The heads of a 2K-token prompt of the paper's 12-head model, as slices of one joint projection.
        _norm("norm_fwd", 1, 2048, 12, 12, 64, fused=True, name="norm_fwd_2k"),
        # A training step's share: four sequences of 8K tokens, the gradients.
        _norm("norm_bwd", 4, 8192, 12, 12, 64, name="norm_bwd_8k_b4"),
        # A float32 user (numerical studies): odd lengths, fewer key heads than query heads, heads of 32.
        _norm("norm_bwd", 3, 1003, 6, 2, 32, "f32", name="norm_bwd_ragged_f32"),
        # One token of each of 64 sequences enters the cache: the smallest call of a serving step.
        _append(64, 12, 12, 64, 64, "1", 100, 2000, False, name="append_decode_b64"),
        # Prompts of up to 8K tokens, heads of 128, shared key heads, normed on the way in.
        _append(3, 16, 4, 128, 64, "2048-8192", 0, 0, True, fused=True, name="append_prompts_d128"),
        # One sequence at 32K tokens decodes a token with the paper's patterns: latency is all there is.
        _attn(1, 12, 12, 64, 64, "1", 32767, 32767, PAPER, name="attn_decode_32k"),
        # 64 sequences of 1K to 32K tokens decode a token each.
        _attn(64, 12, 12, 64, 64, "1", 1000, 32767, PAPER, name="attn_decode_b64"),
        # Dense attention over long caches with four query heads to a key head, heads of 128.
        _attn(8, 16, 4, 128, 128, "1", 8192, 65535, "1048576:1", name="attn_decode_dense_d128"),
        # A 512-token chunk of a long prompt against the 31K tokens before it.
        _attn(1, 12, 12, 64, 64, "512", 31500, 31500, PAPER, name="attn_chunk_512"),
        # A long prompt's chunk of 4096 tokens: an ordinary prefill step.
        _attn(1, 12, 12, 64, 64, "4096", 28672, 28672, PAPER, name="attn_chunk_4k"),
        # A serving step of chunked prefill: one prompt's chunk among sequences that decode.
        _attn(16, 12, 12, 64, 16, "mixed-1000", 500, 8000, "2048:1,4096:2,8192:4", name="attn_mixed_b16"),
        # A float32 check of a small model: odd lengths and patterns, pages of 16, heads of 32.
        _attn(3, 6, 2, 32, 16, "1-300", 0, 1700, "512:1,1777:3,5003:8", "f32", name="attn_ragged_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _patterns(rng):
    """One to six patterns of growing segment length and dilation; now and then without the one that keeps every
    row, and now and then dense."""
    if rng.random() < 0.2:
        return "1048576:1"
    w, r = rng.choice([128, 512, 1024, 2048, 2048, 2048, 4096, rng.randint(100, 3000)]), 1
    a, b = rng.choice([2, 2, 4]), rng.choice([2, 2, 3, 4])
    out = []
    for _ in range(rng.randint(1, 6)):
        out.append((w, min(r, w)))
        w, r = w * a, r * b
    if len(out) > 1 and rng.random() < 0.15:
        out = out[1:]
    return ",".join("%d:%d" % p for p in out)


def draw(rng):
    while True:
        kind = rng.choice(["norm_fwd", "norm_bwd", "append", "attn", "attn", "attn"])
        D = rng.choice([32, 64, 64, 128])
        Hkv = rng.randint(1, 16)
        H = Hkv * rng.choice([1, 1, 1, 2, 3, 4, 8])
        if H > 48:
            continue
        dtype = "f32" if rng.random() < 0.15 else "bf16"
        page = rng.choice([8, 16, 32, 64, 64, 128, 256])
        lengths = rng.randint(1, 10**6)
        if kind.startswith("norm"):
            c = _norm(kind, rng.choice([1, 1, 2, 3]), _log_int(rng, 16, 16384), H, Hkv, D, dtype, rng.random() < 0.5)
        elif kind == "append":
            one = rng.random() < 0.5
            new = "1" if one else "1-%d" % _log_int(rng, 2, 8192)
            B = _log_int(rng, 1, 128) if one else rng.randint(1, 6)
            c = _append(B, H, Hkv, D, page, new, 0, _log_int(rng, 16, 8000 if one else 2000), rng.random() < 0.5,
                        dtype, rng.random() < 0.5, lengths)
            if sum(n + x for n, x in _lengths(c)) * Hkv * D > 1 << 28:
                continue
        else:
            form = rng.choice(["one", "one", "chunk", "mixed"])
            hi = _log_int(rng, 64, 32768)
            lo = rng.choice([0, hi // 8, hi])
            if form == "one":
                B, new = _log_int(rng, 1, 64), "1"
            elif form == "chunk":
                B, new = rng.randint(1, 3), "%d-%d" % (1, _log_int(rng, 2, 4096))
            else:
                B, new = rng.randint(2, 12), "mixed-%d" % _log_int(rng, 16, 1024)
            if dtype == "f32":
                hi, lo = min(hi, 4096), min(lo, 4096)
            c = _attn(B, H, Hkv, D, page, new, lo, hi, _patterns(rng), dtype, lengths)
            lens = _lengths(c)
            S = max(n + x for n, x in lens)
            if B * H * max(n for n, _ in lens) * S > 1.6e9 or B * S * Hkv * D > 1.6e9:
                continue
            if work(c)["flops"] > (2e9 if dtype == "f32" else 3e10):
                continue
        if work(c)["bytes"] <= 4.5e8:
            return c


# ---------------------------------------------------------------------------
# Lengths, work
# ---------------------------------------------------------------------------
def _lengths(case):
    """(new tokens, tokens cached before) of each sequence.  `new`: "n" for all, "lo-hi", or "mixed-n": one
    sequence of n among sequences of one."""
    rng = random.Random(case["lengths"])
    out = []
    for b in range(case["B"]):
        new = case["new"]
        if new.startswith("mixed-"):
            n = int(new[6:]) if b == case["B"] // 2 else 1
        elif "-" in new:
            lo, hi = (int(x) for x in new.split("-"))
            n = rng.randint(lo, hi)
        else:
            n = int(new)
        lo, hi = case["ctx_lo"], case["ctx_hi"]
        out.append((n, _log_int(rng, lo + 1, hi + 1) - 1))
    return out


def _pats(case):
    return [tuple(int(x) for x in p.split(":")) for p in case["patterns"].split(",")]


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    H, Hkv, D, size = case["H"], case["Hkv"], case["D"], _size(case)
    if case["kind"].startswith("norm"):
        x = case["B"] * case["N"] * (H + Hkv) * D
        if case["kind"] == "norm_fwd":  # each element read and written; square, norm, weight, rotation
            return {"bytes": 2 * x * size + 2 * D * size, "flops": 7.0 * x}
        return {"bytes": 3 * x * size + 4 * D * size, "flops": 18.0 * x}
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    if case["kind"] == "append":
        return {"bytes": 2 * T * (H + 2 * Hkv) * D * size + 4 * (3 * len(lens) + 1 + T),
                "flops": (7.0 if case["norm"] else 3.0) * T * (H + Hkv) * D}
    rows = pairs = pages = 0
    for n, ctx in lens:
        seen = np.zeros((Hkv, ctx + n), dtype=bool)
        for w, r in _pats(case):
            for g in range(ctx // w, (ctx + n - 1) // w + 1):
                end = min(ctx + n, (g + 1) * w) - g * w  # segment-local end of the new tokens
                begin = max(ctx - g * w, 0)
                for h in range(H):
                    s = h % r
                    t0, t1 = max(0, -((s - begin) // r)), max(0, -((s - end) // r))  # kept queries [t0, t1)
                    if t1 > t0:
                        pairs += (t1 * (t1 + 1) - t0 * (t0 + 1)) // 2
                        seen[h // (H // Hkv), g * w + s: g * w + s + (t1 - 1) * r + 1: r] = True
        rows += int(seen.sum())
        pages += -(-(ctx + n) // case["page"])
    return {"bytes": 2 * rows * D * size + 2 * T * H * D * size + 4 * T * H + 4 * (pages + 2 * len(lens) + 1),
            "flops": 4.0 * D * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
class _Draw:
    """Seeded Gaussian tensors on the GPU, drawn in chunks."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed * 1000003 + 29)

    def __call__(self, shape, dtype, sigma=1.0, mean=0.0):
        n = math.prod(shape)
        out = torch.empty(n, dtype=dtype, device="cuda")
        for lo in range(0, n, 1 << 27):
            hi = min(n, lo + (1 << 27))
            out[lo:hi] = torch.randn(hi - lo, generator=self.gen, device="cuda").mul_(sigma).add_(mean)
        return out.view(shape)


def _projections(d, lead, case, dtype):
    """q, k, v with the given leading sizes: tensors of their own, or slices of one joint projection's output."""
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    if not case["fused"]:
        return d((*lead, H, D), dtype), d((*lead, Hkv, D), dtype), d((*lead, Hkv, D), dtype)
    x = d((*lead, H + 2 * Hkv, D), dtype)
    return x[..., :H, :], x[..., H: H + Hkv, :], x[..., H + Hkv:, :]


def prepare(case, seed):
    d, dt = _Draw(seed), DTYPES[case["dtype"]]
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    st = {"case": case}
    if case["kind"].startswith("norm") or case.get("norm"):
        st["qw"], st["kw"] = d((D,), dt, 0.2, 1.0), d((D,), dt, 0.2, 1.0)
    if case["kind"].startswith("norm"):
        lead = (case["B"], case["N"])
        st["q"], st["k"], _ = _projections(d, lead, case, dt)
        if case["kind"] == "norm_bwd":
            st["dq"], st["dk"] = d((*lead, H, D), dt), d((*lead, Hkv, D), dt)
        return st
    lens, page = _lengths(case), case["page"]
    T, B = sum(n for n, _ in lens), len(lens)
    blocks = [-(-(n + x) // page) for n, x in lens]
    pages = sum(blocks)
    # the pages of a pool that sequences have come and gone in: in no order
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed), dtype=torch.int64).to(torch.int32)
    table = torch.zeros((B, max(blocks)), dtype=torch.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at: at + n]
        at += n
    st["table"] = table.cuda()
    st["lens"] = torch.tensor([n + x for n, x in lens], dtype=torch.int32, device="cuda")
    st["start"] = torch.tensor(np.cumsum([0] + [n for n, _ in lens]), dtype=torch.int32, device="cuda")
    st["max_new"], st["max_len"] = max(n for n, _ in lens), max(n + x for n, x in lens)
    st["k_cache"], st["v_cache"] = d((pages, Hkv, page, D), dt), d((pages, Hkv, page, D), dt)
    if case["kind"] == "append":
        st["q"], st["k"], st["v"] = _projections(d, (T,), case, dt)
        st["center"] = max(blocks) * page // 2
        return st
    st["q"] = d((T, H, D), dt)
    st["patterns"] = _pats(case)
    return st


# ---------------------------------------------------------------------------
# The calls
# ---------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    if own:
        import paper_2307_02486_amd as da
        if kind == "norm_fwd":
            return da.qk_norm_xpos(st["q"], st["k"], st["qw"], st["kw"])
        if kind == "norm_bwd":
            return da.qk_norm_xpos_bwd(st["dq"], st["dk"], st["q"], st["k"], st["qw"], st["kw"])
        if kind == "append":
            q = da.cache_append(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lens"],
                                st["start"], q_weight=st.get("qw"), k_weight=st.get("kw"), center=st["center"])
            return q, st["k_cache"], st["v_cache"]
        return da.paged_attn(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["start"],
                             st["patterns"], max_new=st["max_new"])
    if kind == "norm_fwd":
        c = _tables(torch.arange(st["q"].shape[1], device="cuda"), st["q"].shape[1] // 2, st["q"].shape[-1])
        return _norm_rotate(st["q"], st["qw"], c, 1), _norm_rotate(st["k"], st["kw"], c, -1)
    if kind == "norm_bwd":
        c = _tables(torch.arange(st["q"].shape[1], device="cuda"), st["q"].shape[1] // 2, st["q"].shape[-1])
        dq, dqw = _norm_rotate_grad(st["dq"], st["q"], st["qw"], c, 1)
        dk, dkw = _norm_rotate_grad(st["dk"], st["k"], st["kw"], c, -1)
        return dq, dk, dqw, dkw
    return _append_plain(st) if kind == "append" else _attn_plain(st)


# ---------------------------------------------------------------------------
# Plain forms: elementary operations in float32, rounded once at the end
# ---------------------------------------------------------------------------
def _tables(pos, center, D):
    """cos, sin and the two scales [..., 1, D/2] of each position.  The angles, up to tens of thousands of
    radians, are formed in float64: a float32 product would be off by a thousandth of a radian."""
    i = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    a = pos.to(torch.float64)[..., None, None] * BASE ** (-2 * i / D)
    zeta = torch.log2((2 * i / D + GAMMA) / (1 + GAMMA)).float()
    e = ((pos - center).float() / SCALE_BASE)[..., None, None] * zeta
    return a.cos().float(), a.sin().float(), torch.exp2(e), torch.exp2(-e)


def _rotate(x, tables, sign):
    cos, sin, up, down = tables
    s = up if sign > 0 else down
    y0 = s * (x[..., 0::2] * cos - x[..., 1::2] * sin)
    y1 = s * (x[..., 0::2] * sin + x[..., 1::2] * cos)
    return torch.stack((y0, y1), dim=-1).flatten(-2)


def _norm_rotate(x, weight, tables, sign):
    f = x.float()
    if weight is not None:
        f = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * weight.float()
    return _rotate(f, tables, sign).to(x.dtype)


def _norm_rotate_grad(dy, x, weight, tables, sign):
    cos, sin, up, down = tables
    dn = _rotate(dy.float(), (cos, -sin, up, down), sign)  # the transpose
    f = x.float()
    rstd = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    xhat = f * rstd
    dw = (dn * xhat).flatten(0, 2).sum(0)
    dxhat = dn * weight.float()
    dx = rstd * (dxhat - xhat * (dxhat * xhat).mean(-1, keepdim=True))
    return dx.to(x.dtype), dw.to(x.dtype)


def _sequences(st):
    """Sequence and position of each new token."""
    tok = torch.arange(st["q"].shape[0], device="cuda")
    seq = torch.searchsorted(st["start"][1:].long(), tok, right=True)
    n = (st["start"][1:] - st["start"][:-1]).long()
    return seq, st["lens"].long()[seq] - n[seq] + tok - st["start"].long()[seq]


def _append_plain(st):
    seq, pos = _sequences(st)
    page = st["case"]["page"]
    tables = _tables(pos, st["center"], st["case"]["D"])
    where = st["table"].long()[seq, pos // page]
    st["k_cache"][where, :, pos % page] = _norm_rotate(st["k"], st.get("kw"), tables, -1)
    st["v_cache"][where, :, pos % page] = st["v"]
    return _norm_rotate(st["q"], st.get("qw"), tables, 1), st["k_cache"], st["v_cache"]


def _attn_plain(st):
    """Every cached key against every new token, each weighted by the number of patterns that hold the pair."""
    case = st["case"]
    B, H, Hkv, D = case["B"], case["H"], case["Hkv"], case["D"]
    Q, S = st["max_new"], st["max_len"]
    seq, pos = _sequences(st)
    row = torch.arange(st["q"].shape[0], device="cuda") - st["start"].long()[seq]
    q = torch.zeros((B, Q, H, D), device="cuda")
    q[seq, row] = st["q"].float()
    at = torch.full((B, 1, Q, 1), -1, dtype=torch.int32, device="cuda")
    at[seq, 0, row, 0] = pos.to(torch.int32)
    q = q.permute(0, 2, 1, 3).reshape(B, Hkv, H // Hkv * Q, D)

    def cached(cache):  # [B, Hkv, S, D]
        return cache[st["table"].long()].permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :S].float()

    s = (q @ cached(st["k_cache"]).transpose(-1, -2)).view(B, H, Q, S) * D ** -0.5
    key = torch.arange(S, device="cuda", dtype=torch.int32)
    head = torch.arange(H, device="cuda", dtype=torch.int32)[:, None, None]
    count = torch.zeros((B, H, Q, S), device="cuda")
    for w, r in st["patterns"]:
        off = head % r
        kept_q, kept_k = (at % w) % r == off, (key % w) % r == off
        count += (at // w == key // w) & kept_q & kept_k
    count *= (key <= at) & (at >= 0)
    s = s.masked_fill(count == 0, -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(s - m) * count
    den = p.sum(-1, keepdim=True)
    o = (p / den.clamp_min(1e-37)).view(B, Hkv, H // Hkv * Q, S) @ cached(st["v_cache"])
    o = o.view(B, H, Q, D).permute(0, 2, 1, 3)[seq, row]
    lse = (m + torch.log(den))[..., 0].permute(0, 2, 1)[seq, row]
    return o.to(st["q"].dtype), lse.t().contiguous()


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def _xpos64(x, pos, center, sign):
    """x [..., heads, D] float64 at positions [...]: the pairs as complex numbers times s e^(i a)."""
    D = x.shape[-1]
    i = torch.arange(D // 2, dtype=torch.float64, device=x.device)
    ang = pos.double().unsqueeze(-1) * torch.pow(torch.tensor(BASE, dtype=torch.float64, device=x.device), -2 * i / D)
    zeta = (2 * i / D + GAMMA) / (1 + GAMMA)
    mag = torch.pow(zeta, sign * (pos.double().unsqueeze(-1) - center) / SCALE_BASE)
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], D // 2, 2).contiguous()) * torch.polar(mag, ang).unsqueeze(-2)
    return torch.view_as_real(z).reshape(x.shape)


def _heads64(x, w, pos, center, sign):
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w
    return _xpos64(x, pos, center, sign)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("norm"):
        pos = torch.arange(case["N"], device="cuda").expand(case["B"], case["N"])
        outs, grads = [], []
        for x, w, dy, sign in (("q", "qw", "dq", 1), ("k", "kw", "dk", -1)):
            x64 = st[x].double().requires_grad_(case["kind"] == "norm_bwd")
            w64 = st[w].double().requires_grad_(case["kind"] == "norm_bwd")
            y = _heads64(x64, w64, pos, case["N"] // 2, sign)
            outs.append(y)
            if case["kind"] == "norm_bwd":
                grads.append(torch.autograd.grad(y, (x64, w64), st[dy].double()))
        return tuple(outs) if not grads else (grads[0][0], grads[1][0], grads[0][1], grads[1][1])
    lens, page, D = _lengths(case), case["page"], case["D"]
    if case["kind"] == "append":
        kc, vc, qo, at = st["k_cache"].double(), st["v_cache"].double(), [], 0
        w = [None if st.get(n) is None else st[n].double() for n in ("qw", "kw")]
        for b, (n, ctx) in enumerate(lens):
            pos = torch.arange(ctx, ctx + n, device="cuda")
            qo.append(_heads64(st["q"][at: at + n].double(), w[0], pos, st["center"], 1))
            k = _heads64(st["k"][at: at + n].double(), w[1], pos, st["center"], -1)
            pages = st["table"][b].long()[torch.div(pos, page, rounding_mode="floor")]
            kc[pages, :, pos % page], vc[pages, :, pos % page] = k, st["v"][at: at + n].double()
            at += n
        return torch.cat(qo), kc, vc
    # attention: pattern by pattern and segment by segment on explicit index sets, then mixed by denominators
    H, G = case["H"], case["H"] // case["Hkv"]
    T = st["q"].shape[0]
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, ctx) in enumerate(lens):
        pages = st["table"][b, : -(-(ctx + n) // page)].long()
        keys, vals = (st[c][pages].transpose(1, 2).flatten(0, 1) for c in ("k_cache", "v_cache"))
        q = st["q"][at: at + n]
        for w, r in _pats(case):
            for g in range(ctx // w, (ctx + n - 1) // w + 1):
                for s in range(min(r, H)):
                    end = min((g + 1) * w, ctx + n)
                    rows = torch.arange(min(g * w + s, end), end, r, device="cuda")
                    new = rows[rows >= ctx]
                    if not new.numel():
                        continue
                    heads = torch.arange(s, H, r, device="cuda")
                    for part in new.split(1024):
                        qs = q[part - ctx][:, heads].double().transpose(0, 1)
                        ks = keys[rows][:, heads // G].double().permute(1, 2, 0)
                        sc = qs @ ks / math.sqrt(D)
                        sc.masked_fill_(rows[None, None, :] > part[None, :, None], -math.inf)
                        l = torch.logsumexp(sc, -1)
                        o = torch.softmax(sc, -1) @ vals[rows][:, heads // G].double().transpose(0, 1)
                        i, j = (part - ctx + at)[:, None], heads[None, :]
                        both = torch.logaddexp(lse[i, j], l.t())
                        out[i, j] = out[i, j] * torch.exp(lse[i, j] - both)[..., None] \
                            + o.transpose(0, 1) * torch.exp(l.t() - both)[..., None]
                        lse[i, j] = both
        at += n
    return out, lse.t().contiguous()
