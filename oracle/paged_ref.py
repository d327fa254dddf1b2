"""Float64 references of serving from a paged cache and of the head norms:
each new token's keys found one by one from the definition (segment, residue,
position), no segment-wise algorithm; and RMS norm with xPos on complex pairs."""
import numpy as np


def counts(pos, keys, H, patterns):
    """[H, keys]: how many patterns let a query at position pos see each key."""
    pos, key = int(pos), np.arange(keys)
    out = np.zeros((H, keys))
    for w, r in patterns:
        for h in range(H):
            if (pos % w) % r == h % r:  # w and r beyond any position act like one past the last
                W, R = min(w, keys + H), min(r, keys + H)
                out[h] += (key // W == pos // W) & ((key % W) % R == h % R) & (key <= pos)
    return out


def paged_attention_ref(q, k, v, first, patterns, scale=None):
    """One sequence: q [n, H, D] at positions first .. first + n - 1, k and v
    [length, Hkv, D].  Returns out [n, H, D] and lse [n, H]; a row without keys
    has zeros and -inf."""
    n, H, D = q.shape
    group = H // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out, lse = np.zeros(q.shape), np.full((n, H), -np.inf)
    for i in range(n):
        c = counts(first + i, k.shape[0], H, patterns)
        for h in range(H):
            sel = np.flatnonzero(c[h])
            if not sel.size:
                continue
            s = scale * (k[sel, h // group] @ q[i, h])
            m = s.max()
            p = c[h, sel] * np.exp(s - m)
            out[i, h] = p @ v[sel, h // group] / p.sum()
            lse[i, h] = m + np.log(p.sum())
    return out, lse


def heads_ref(x, weight, pos, sign, center, base=10000.0, gamma=0.4, scale_base=512.0, eps=1e-6):
    """RMS norm with weight (or None: no norm), then xPos, of x [..., heads, D] at positions [...]."""
    D = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    i = np.arange(D // 2)
    zeta = (2 * i / D + gamma) / (1 + gamma)
    pos = np.asarray(pos, np.float64)[..., None, None]
    turn = zeta ** (sign * (pos - center) / scale_base) * np.exp(1j * pos * base ** (-2 * i / D))
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * turn
    y = np.empty(x.shape)
    y[..., 0::2], y[..., 1::2] = z.real, z.imag
    return y


def heads_bwd_ref(dy, x, weight, pos, sign, center, base=10000.0, gamma=0.4, scale_base=512.0, eps=1e-6):
    """Gradients (dx, dweight) of heads_ref with a norm: the transposed rotation
    is a product with the conjugate, the norm's derivative a projection."""
    D = x.shape[-1]
    i = np.arange(D // 2)
    zeta = (2 * i / D + gamma) / (1 + gamma)
    p = np.asarray(pos, np.float64)[..., None, None]
    turn = zeta ** (sign * (p - center) / scale_base) * np.exp(-1j * p * base ** (-2 * i / D))
    z = (dy[..., 0::2] + 1j * dy[..., 1::2]) * turn
    dn = np.empty(x.shape)
    dn[..., 0::2], dn[..., 1::2] = z.real, z.imag
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xhat, g = x / rms, dn * weight
    dx = (g - xhat * (g * xhat).mean(-1, keepdims=True)) / rms
    return dx, (dn * xhat).reshape(-1, D).sum(0)
