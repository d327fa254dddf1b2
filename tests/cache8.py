"""Caches in 8 bits for the tests: pools of random values, their read-out, and the
append of the reference block by block."""
import numpy as np
import torch

from oracle.compressed_ref import BLOCK, append_block

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def blocks_of(page):
    return page // min(page, BLOCK)


def pool(pages, Hkv, page, D, seed, device="cuda", spread=3):
    """(values, scales) at random: finite e4m3 bytes, scales over 2^+-spread around 2^-9."""
    rng = np.random.default_rng(seed)
    b = rng.integers(0, 127, (pages, Hkv, page, D)) + 128 * rng.integers(0, 2, (pages, Hkv, page, D))
    s = 118 + rng.integers(-spread, spread + 1, (pages, Hkv, blocks_of(page)))
    return torch.from_numpy(b.astype(np.uint8)).to(device).view(F8), torch.from_numpy(s.astype(np.uint8)).to(device).view(E8)


def normal_pool(pages, Hkv, page, D, seed, device="cuda"):
    """(values, scales) of Gaussian rows, as an append leaves them."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(pages, Hkv, blocks_of(page), min(page, BLOCK), D)).astype(np.float32)
    e = np.ceil(np.log2(np.abs(x).max((-1, -2)) / 448)).astype(np.int32)
    v = torch.from_numpy(np.ldexp(x, -e[..., None, None])).to(F8).view(torch.uint8).reshape(pages, Hkv, page, D)
    return v.to(device).view(F8), torch.from_numpy((e + 127).astype(np.uint8)).to(device).view(E8)


def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def unscaled(t):
    """The e4m3 values in float64."""
    return t.cpu().double().numpy()


def elements(vals, scale):
    """The cache's elements [pages, Hkv, page, D] in float64."""
    e = bytes_of(scale).astype(np.float64) - 127
    return unscaled(vals) * np.exp2(np.repeat(e, vals.shape[2] // scale.shape[2], axis=2))[..., None]


def append_ref(vals, exps, table, lens, start, new, page):
    """New rows [T, Hkv, D] (float64) into vals [pages, Hkv, page, D] (e4m3 values)
    and exps [pages, Hkv, blocks], in place."""
    pages, Hkv, _, _ = vals.shape
    size = min(page, BLOCK)
    for b in range(len(lens)):
        n = int(start[b + 1] - start[b])
        c0, c1 = int(lens[b]) - n, int(lens[b])
        for lo in range(c0 // size * size, c1, size):
            p, at = int(table[b, lo // page]), lo % page
            if not 0 <= p < pages:
                continue
            t0, t1 = max(lo, c0), min(lo + size, c1)
            rows = new[start[b] + t0 - c0: start[b] + t1 - c0]
            for h in range(Hkv):
                got, e = append_block(vals[p, h, at: at + t0 - lo], int(exps[p, h, at // size]), rows[:, h])
                vals[p, h, at: at + t1 - lo], exps[p, h, at // size] = got, e


def rows_of(values, table_row, page, length):
    """A sequence's rows [length, Hkv, D] from a pool's, and whether each one's page is there."""
    at = np.arange(length)
    p = table_row[at // page].astype(np.int64)
    there = (p >= 0) & (p < values.shape[0])
    x = values[np.where(there, p, 0), :, at % page]
    return np.where(there[:, None, None], x, 0.0), there
