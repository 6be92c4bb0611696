"""What the serving operators' tests share: inputs, tolerances, comparison."""
import numpy as np

# Half a rounding step relative to the value.
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def tolerances(ref, dtype, d, n):
    """Elementwise bounds of |o - o*| and |lse - lse*| for rows over at most n keys of width d.

    Logits: d products and sums and two scalings in float32, so each is off by
    at most dz = (d + 4) 2^-24 sum_c |q_c k_c| |scale|, and its exponential's
    argument by another 4 units of 2^-24 (1 + |z|) (a product, a difference,
    the exponential), with |z| <= the same sum.  Weights are then off by a
    factor of 1 +- dp, dp = 2 (dz + 4 2^-24 (1 + dots)); their sums and the
    sums over values add n + 16 float32 roundings (16: rescalings, joins of
    parts).  bf16: each weight and the result are rounded once to bf16.

    The last term is what underflow can lose.  A weight, relative to a maximum
    that is at most the row's largest logit, so that the weights' sum is at
    least 1, is flushed to zero below float32's and bf16's least normal value
    2^-126; in the cache this goes for the weight times its block's value
    scale.  What multiplies it is a value (below 2^9 in these tests) or a code
    (at most 448 < 2^9), so each of n keys loses at most 2^-126 2^9.
    """
    u = 2.0 ** -24
    dp = 2 * ((d + 4) * u * ref["dots"] + 4 * u * (1 + ref["dots"]))
    rel = dp + (n + 16) * u + (HALF["bf16"] if dtype == "bf16" else 0.0)
    tol_o = rel[..., None] * ref["abs_o"] * (1 + 2.0 ** -7) + HALF[dtype] * np.abs(ref["o"]) * (1 + 2.0 ** -7) + n * 2.0 ** -117
    lse = np.where(np.isfinite(ref["lse"]), ref["lse"], 0)
    tol_lse = dp + (n + 16) * u + 4 * u * np.abs(lse)
    return tol_o, tol_lse


def check(out_o, out_lse, ref, dtype, d, n, what=""):
    o, lse = np.asarray(out_o, np.float64), np.asarray(out_lse, np.float64)
    tol_o, tol_lse = tolerances(ref, dtype, d, n)
    fin = np.isfinite(ref["o"])
    assert np.array_equal(np.isfinite(o), fin), (what, "where o is finite", int((np.isfinite(o) != fin).sum()))
    worst = float(np.max(np.where(fin, np.abs(np.where(fin, o, 0) - np.where(fin, ref["o"], 0)) / tol_o, 0), initial=0))
    assert worst <= 1, (what, "o", worst)
    fl = np.isfinite(ref["lse"])
    assert np.array_equal(lse[~fl & ~np.isnan(ref["lse"])], ref["lse"][~fl & ~np.isnan(ref["lse"])]), (what, "infinite lse")
    wl = float(np.max(np.where(fl, np.abs(np.where(fl, lse, 0) - np.where(fl, ref["lse"], 0)) / tol_lse, 0), initial=0))
    assert wl <= 1, (what, "lse", wl)
    return worst, wl


def rows(rng, shape, outliers=True):
    """Standard normal rows, four channels of them scaled by 8."""
    x = rng.standard_normal(shape).astype(np.float32)
    if outliers and shape[-1] >= 8:
        x[..., rng.permutation(shape[-1])[:4]] *= 8
    return x
