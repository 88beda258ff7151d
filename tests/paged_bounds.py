"""Bounds on attention outputs relative to the outputs themselves.

A weight's relative error d_n depends on the queries and keys alone, so with
values that are independent of them and have mean zero an output's error
sum w_n d_n (V_n - o) has a norm of at most max|d| sqrt(sum w_n^2 |V_n|^2), and
the output itself one of about sqrt(sum w_n^2 |V_n|^2): the ratio of the norms
is at most max|d|, however many keys there are.  (An absolute bound from the
largest value is wider than the outputs where thousands of keys share the
weight.)  The ratio of one row of 128 channels scatters by about 1 / sqrt(128)
around that, of all rows together by far less.
"""
from __future__ import annotations

D = 128


def logit_error(q, k, scale):
    """Bound on the error of any logit: 128 exact products summed in float32 and
    up to four factors, of the largest sum of magnitudes.  q [n, Hq, D], k
    [Hkv, N, D] torch tensors."""
    g = q.shape[1] // k.shape[0]
    big = 0.0
    for h in range(q.shape[1]):
        big = max(big, float((q[:, h].float().abs() @ k[h // g].float().abs().T.contiguous()).max()))
    return scale * big * 132 * 2.0 ** -24


def relative_bound(q, k, scale, rows, sums):
    """rows: query rows of a KV head (up to 16 the weights are a high + low bf16
    pair); sums: float32 additions in a row on the way of a value into the output."""
    return logit_error(q, k, scale) + (2.0 ** -16 if rows <= 16 else 2.0 ** -8) + (sums + 32) * 2.0 ** -24


def outputs_agree(out, want, rel):
    """Whether out [n, Hq, D] is within rel of want: as a whole, and every row
    within twice that."""
    off = out.double() - want
    whole = float(off.norm()) <= 1.1 * rel * float(want.norm())
    return whole and bool((off.norm(dim=-1) <= 2 * rel * want.norm(dim=-1)).all())
