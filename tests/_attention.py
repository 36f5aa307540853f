"""Error bounds of the attention tests, from the arithmetic that the calls document.

u is half a step of fp32 relative to the value (2^-24), b of bf16 (2^-8).
A score is a sum of d products (d half steps of the sum of magnitudes ``arg``, and
four more for the scale, the fused multiply-add of the exponent and its argument's
rounding), and the base-2 exponential adds two: a weight is off by the factor
1 + delta, delta = 2 ((d + 4) arg + 4) u, where the 2 is numerator and denominator.
Sums over t keys add (t + 8) u of their magnitude ``mag``, which also covers the
rescaling of split ranges.  In bf16 each weight is rounded once before the second
product and the result once after it.
"""

import numpy as np

U32, UB = 2.0 ** -24, 2.0 ** -8


def bounds(ref, d, t, dtype, mag=None, arg=None):
    """(bound of out [n, H_q, d], of lse [n, H_q])."""
    mag = ref["mag"] if mag is None else mag
    arg = ref["arg"] if arg is None else arg
    delta = 2 * ((d + 4) * arg + 4) * U32
    err = mag * (delta[..., None] + (t + 8) * U32)
    if dtype == "bf16":
        err = err + UB * mag
        err = err + UB * (np.abs(ref["out"]) + err)
    else:
        err = err + U32 * np.abs(ref["out"])
    with np.errstate(invalid="ignore"):
        lse = delta / 2 + (t + 8) * U32 + 4 * U32 * np.abs(np.where(np.isinf(ref["lse"]), 0, ref["lse"]))
    return err, lse


def check(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: infinities"
    off = np.abs(got - np.where(fine, want, 0))[fine]
    over = off > np.broadcast_to(bound, want.shape)[fine]
    assert not over.any(), (f"{what}: {int(over.sum())} of {over.size} off by more than the bound, "
                            f"worst {float((off / np.maximum(np.broadcast_to(bound, want.shape)[fine], 1e-300)).max()):.2f} of it")


def logical(table, page_codes, H, d, P, b, t):
    """Codes [2, t, H, d], s and o [2, t, H, d/32] of the first t tokens of sequence b, and
    which of them are in a page; page_codes: a dict of unpacked pages."""
    c = np.zeros((2, t, H, d), np.int64)
    s = np.zeros((2, t, H, d // 32), np.float32)
    o = np.zeros((2, t, H, d // 32), np.float32)
    seen = np.zeros(t, bool)
    for j in range(-(-t // P)):
        p = int(table[b][j])
        if p not in page_codes:
            continue
        n = min(P, t - j * P)
        at = slice(j * P, j * P + n)
        c[:, at], s[:, at], o[:, at] = (x[:, :n] for x in page_codes[p])
        seen[at] = True
    return c, s, o, seen
