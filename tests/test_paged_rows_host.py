"""The bars of paged_rows on the CPU: a row of the other oracle is within them, and
mistakes in V's rows, planted in the oracle, are not.  No GPU."""
import numpy as np
import pytest

from oracle.paged_ref import paged_attention_ref
from tests.paged_rows import row


@pytest.mark.parametrize("patterns", [[(64, 1), (256, 3)], [(1 << 20, 1)], [(32, 1), (32, 1), (96, 2)]], ids=str)
def test_rows_are_the_definition(patterns):
    rng = np.random.default_rng(4)
    q, k, v = rng.normal(size=(3, 4, 16)), rng.normal(size=(300, 2, 16)), rng.normal(size=(300, 2, 16))
    out, lse = paged_attention_ref(q, k, v, 297, patterns)
    for i in range(3):
        for h in range(4):
            o, l, bar = row(q[i, h], k[:, h // 2], v[:, h // 2], 297 + i, h, patterns)
            assert np.allclose(o, out[i, h], atol=1e-12) and (bar >= 0).all()
            assert l == lse[i, h] == -np.inf or abs(l - lse[i, h]) <= 1e-12


@pytest.mark.parametrize("mistake", ["32 rows of another place", "a tile of 64 zeroed", "a tile of 32 in reverse"])
@pytest.mark.parametrize("keys, D", [(2500, 64), (5001, 64), (8500, 128), (5200, 32)])
def test_a_tile_of_values_in_the_wrong_place_shows(keys, D, mistake):
    for seed in range(4):
        rng = np.random.default_rng(seed)
        q, k, v = rng.normal(size=D), rng.normal(size=(keys, D)), rng.normal(size=(keys, D))
        bad, at = v.copy(), int(rng.integers(0, keys - 200))
        if mistake.startswith("32"):
            bad[at: at + 32] = v[at + 100: at + 132]
        elif mistake.startswith("a tile of 64"):
            bad[at: at + 64] = 0
        else:
            bad[at: at + 32] = v[at: at + 32][::-1]
        out, _, bar = row(q, k, v, keys - 1, 0, [(1 << 20, 1)], bad)
        ref = row(q, k, v, keys - 1, 0, [(1 << 20, 1)])[0]
        assert (np.abs(out - ref) > bar).sum() > D // 16, seed
