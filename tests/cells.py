"""What the tests of cells that share blocks have in common: states and their comparison."""
import numpy as np

from oracle.serving import E4M3


def cache_arrays(rng, n_blocks, bs, d, dp, spread=3):
    """A filled cache: every code but NaN, rows and columns past d zero, exponents around 120."""
    k = rng.integers(0, 256, (n_blocks, bs, dp)).astype(np.uint8)
    v = rng.integers(0, 256, (n_blocks, dp, bs)).astype(np.uint8)
    for x in (k, v):
        x[(x & 0x7F) == 0x7F] = 0
    k[:, :, d:] = 0
    v[:, d:] = 0
    e = lambda: rng.integers(120 - spread, 121 + spread, n_blocks).astype(np.uint8)
    return dict(k=k, v=v, k_exp=e(), v_exp=e(), d=d)


def random_state(rng, lens, bs, dp, d, W=None, n_blocks=None, spread=3):
    """Cells of these lengths in blocks of no order; none shared."""
    need = [-(-int(n) // bs) for n in lens]
    W = W or max(1, max(need))
    n_blocks = n_blocks or sum(need) + 5
    ids, at = rng.permutation(n_blocks), 0
    table = np.full((len(lens), W), -1, np.int32)
    for c, m in enumerate(need):
        table[c, :m] = ids[at:at + m]
        at += m
    free = np.concatenate([ids[at:], np.full(at, -7)]).astype(np.int32)
    return dict(cache_arrays(rng, n_blocks, bs, d, dp, spread), table=table, lens=np.array(lens, np.int32), free_list=free,
                n_free=n_blocks - at, shared=np.zeros(n_blocks, np.int32))


def same_codes(got, want):
    """Codes of equal values (a NaN has two codes, and so has zero)."""
    a, b = E4M3[got], E4M3[want]
    return (got == want) | (a == b) | (np.isnan(a) & np.isnan(b))


def compare(got, want, was, what=""):
    """A state after a call: whole numbers equal, codes of the same values, and the same bytes where nothing changed."""
    for key in ("table", "lens", "shared", "k_exp", "v_exp"):
        assert np.array_equal(got[key], want[key]), (what, key)
    n = want["n_free"]
    assert got["n_free"] == n and np.array_equal(got["free_list"][:n], want["free_list"][:n]), (what, "stack")
    for key in ("k", "v"):
        assert same_codes(got[key], want[key]).all(), (what, key, int((~same_codes(got[key], want[key])).sum()))
        still = (want[key] == was[key]).reshape(len(was[key]), -1).all(1) & (want[key + "_exp"] == was[key + "_exp"])
        assert np.array_equal(got[key][still], was[key][still]), (what, key, "blocks that nothing touched")
