"""Float64 references of serving from a compressed cache, by the definitions:
rounding to e4m3 by counting in units, a block's scale by trying powers of two,
the attention and the pages' weights key by key, eviction by sorting."""
import numpy as np

from .paged_ref import counts

BLOCK = 16


def e4m3(x):
    """x to the nearest value of e4m3, ties to even: whole multiples of 2^-9 below
    2^-6, of an eighth of the leading power of two above."""
    x = np.asarray(x, np.float64)
    lead = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))))
    lead = np.where(lead > np.maximum(np.abs(x), 2.0 ** -6), lead / 2, lead)
    return np.rint(x / (lead / 8)) * (lead / 8)


def block_exponent(amax):
    """The least e >= -126 with amax <= 448 * 2^e."""
    e = -126
    while amax > 448 * 2.0 ** e:
        e += 1
    return e


def append_block(values, e, new):
    """A block of one head with the elements' e4m3 values [old, D] at exponent e
    (not looked at without old rows) and new rows [n, D]: the values [old + n, D]
    and the exponent after the append.  Infinities and NaN become NaN."""
    fin = np.isfinite(new)
    e2 = block_exponent(np.abs(np.where(fin, new, 0.0)).max(initial=0.0))
    if len(values):
        e2 = max(e2, e)
        values = e4m3(values * 2.0 ** (e - e2))
    with np.errstate(invalid="ignore"):
        return np.concatenate([values, np.where(fin, e4m3(np.where(fin, new, 0.0) * 2.0 ** -e2), np.nan)]), e2


def seen(first, n, keys, H, patterns, there):
    """[n, H, keys]: how many patterns let the query at first + i see each key that is there."""
    return np.array([counts(first + i, keys, H, patterns) * there for i in range(n)])


def attention_ref(q, k, v, first, patterns, there, scale=None):
    """One sequence: q [n, H, D] at positions first .., k and v [length, Hkv, D],
    `there` [length] whether a key's page is.  Returns out [n, H, D], lse [n, H]."""
    n, H, D = q.shape
    group, scale = H // k.shape[1], D ** -0.5 if scale is None else scale
    out, lse = np.zeros(q.shape), np.full((n, H), -np.inf)
    c = seen(first, n, k.shape[0], H, patterns, there)
    for i in range(n):
        for h in range(H):
            sel = np.flatnonzero(c[i, h])
            if sel.size:
                s = scale * (k[sel, h // group] @ q[i, h])
                p = c[i, h, sel] * np.exp(s - s.max())
                out[i, h], lse[i, h] = p @ v[sel, h // group] / p.sum(), s.max() + np.log(p.sum())
    return out, lse


def key_weights_ref(q, k, first, patterns, there, lse, scale=None):
    """[length]: what each key of a sequence gets from all rows, given their lse [n, H]."""
    n, H, D = q.shape
    group, scale = H // k.shape[1], D ** -0.5 if scale is None else scale
    c, out = seen(first, n, k.shape[0], H, patterns, there), np.zeros(k.shape[0])
    for i in range(n):
        for h in range(H):
            sel = np.flatnonzero(c[i, h])
            if sel.size and np.isfinite(lse[i, h]):
                out[sel] += c[i, h, sel] * np.exp(scale * (k[sel, h // group] @ q[i, h]) - lse[i, h])
    return out


def evict_ref(weights, table, lens, page, keep, first, last):
    """(table, freed, count) of evict_pages, numpy arrays."""
    table = table.copy()
    freed, count = np.full(table.shape, -1, table.dtype), np.zeros(len(lens), table.dtype)
    for b, n in enumerate(lens):
        end = min(-(-max(int(n), 0) // page), table.shape[1])
        held = [j for j in range(end) if 0 <= table[b, j] < len(weights)]
        may = [j for j in held if first <= j < end - last]
        heavy = lambda j: np.inf if np.isnan(weights[table[b, j]]) else weights[table[b, j]]  # noqa: E731
        nan = lambda j: bool(np.isnan(weights[table[b, j]]))  # noqa: E731
        out = sorted(sorted(may, key=lambda j: (nan(j), heavy(j), j))[: max(0, len(held) - keep)])
        freed[b, : len(out)], count[b] = table[b, out], len(out)
        table[b, out] = -1
    return table, freed, count
