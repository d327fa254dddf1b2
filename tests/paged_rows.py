"""Single rows of attention over a cache in float64, with the error that bf16
arithmetic may leave in each element.

A row's out is sum_i p_i v_i over its keys, p_i the softmax of its scores times
the number of patterns that hold key i.  In bf16:
  * each p_i is rounded to bf16 for the product: an error of at most 2^-8 p_i,
    of standard deviation at most 2^-8 p_i / sqrt(3), independent from key to key;
    six deviations of their sum are 3.5 * 2^-8 sqrt(sum p_i^2 v_i^2);
  * rows of tiles are kept in fp16, within 2^-11 of the largest element of a
    partial row: 2^-11 times the mean of those over the patterns' weights, times 4
    for the splits (at most 16, each of whose rows is larger by the root of their number);
  * float32 sums, scores and exponentials: 2e-5 sum p_i |v_i|;
  * out itself is rounded: 2^-8 |out|.
With thousands of keys that is far below the size of an element, so that a tile of
keys in the wrong place shows."""
import numpy as np


def key_counts(pos, keys, head, patterns):
    """How many patterns let the query at pos of this head see each key."""
    pos, key, c = int(pos), np.arange(keys), []
    for w, r in patterns:
        if (pos % w) % r == head % r:
            c.append((key // w == pos // w) & ((key % w) % r == head % r) & (key <= pos))
        else:
            c.append(np.zeros(keys, bool))
    return np.array(c)


def row(q, k, v, pos, head, patterns, v_seen=None):
    """q [D], k and v [length, D] in float64: out, lse and the bar of each element.
    v_seen: other values that the row is formed with (a mistake, for the tests'
    own test)."""
    c = key_counts(pos, k.shape[0], head, patterns)
    sel = np.flatnonzero(c.any(0))
    if not sel.size:
        return np.zeros(q.shape), -np.inf, np.zeros(q.shape)
    s = k[sel] @ q * q.shape[0] ** -0.5
    e = np.exp(s - s.max())
    each = c[:, sel] * e  # by pattern
    den = each.sum()
    p, vs = each.sum(0) / den, v[sel]
    out = p @ (vs if v_seen is None else v_seen[sel])
    kept = 0.0
    for x in each:
        if x.any():
            kept += np.abs(x @ vs).max() / den
    ref = p @ vs
    bar = 3.5 * 2.0 ** -8 * np.sqrt((p * p) @ (vs * vs)) + 4 * 2.0 ** -11 * kept + 2e-5 * p @ np.abs(vs) \
        + 2.0 ** -8 * np.abs(ref)
    return out, s.max() + np.log(den), bar
