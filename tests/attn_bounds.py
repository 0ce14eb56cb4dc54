"""How far float32 attention may be from its value in 64 bits, from its roundings.

u = 2^-24 is half a float32 step.  A logit is a sum of 128 products and a scale:
off by at most 140 u * size, size the largest sum |q_i k_i| * scale (delta below).
A weight is then off by 2 delta (its own logit and the sum's), two steps of the
exponential, and the n terms of the sums, each rescaled at most as often as the
maximum grows: (3 n + 32) u.  bfloat16 inputs round each weight once to bfloat16,
2^-8 of it.  A result is off by those fractions of the weighted mean of |v|
(`mass`); a bfloat16 result by another 2^-8 of itself.
"""
import numpy as np

U = 2.0 ** -24


def attention_bounds(out, mass, lse, size, n, bf16_in, bf16_out):
    delta = 140 * U * size
    frac = 2 * delta + (3 * n + 32) * U + (2.0 ** -8 if bf16_in else 0.0)
    tol = frac[:, None] * mass
    if bf16_out:
        tol = tol + 2.0 ** -8 * (np.abs(out) + tol)
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return tol + 1e-37, delta + (3 * n + 32) * U + 4 * U * finite


def check_attention(got, got_lse, want, bf16_in, bf16_out, n):
    """got [rows][d] against want = oracle.blocks.masked_attention's (out, lse, mass, size)."""
    out, lse, mass, size = want
    tol, tol_lse = attention_bounds(out, mass, lse, size, n, bf16_in, bf16_out)
    nan = np.isnan(out)
    assert np.array_equal(np.isnan(got), nan), "NaN in other places"
    err = np.where(nan, 0.0, np.abs(got - out))
    assert np.all(err <= np.where(nan, 1.0, tol)), f"off by {(err / np.where(nan, 1.0, tol)).max():.3g} of the bound"
    if got_lse is not None:
        dead = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse), dead), "lse of rows that see nothing"
        live = ~dead & ~np.isnan(lse)
        assert np.array_equal(np.isnan(got_lse), np.isnan(lse))
        assert np.all(np.abs(got_lse[live] - lse[live]) <= tol_lse[live]), "lse"
    return float((err / np.where(nan, 1.0, tol)).max()) if err.size else 0.0
