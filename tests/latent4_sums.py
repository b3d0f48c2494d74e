"""What attention over the 4-bit cache adds to a sequence's sums of weights, held to the oracle in three ways: token by
token to the oracle's bound, which takes every rounding at its largest; in the norm; and in total.

In the norm: a score's operands are rounded to fp16, each off by at most HALF of itself and evenly spread, so that the
score is off by scale HALF / sqrt(3) sqrt(sum of its squared products) a rounded operand. With queries of size 1.5 and
rows of size 1 that is at most 1.2 HALF over both operands, whatever the dimensions, and a weight is off by as much of
itself. 8 HALF holds it, and is less than half of 1 / 128, what a head of 128 that is left out takes away.

In total: a row's weights over all tokens and heads add up to its heads, whatever the operands were rounded to, as both
launches form a score by the same instructions from the same operands in the same order. What is left, in units of
SINGLE, of the whole, with M the largest score times log2(e):
  the exponent's arguments, a rounding of up to 2 M + 15 in either launch, and ln 2 of it:    1.4 (2 M + 15)
  the references, four roundings of up to M + 7 between the launches:                         2.8 (M + 7)
  exponentials (2 each): a weight's in either launch, a partial result's:                     6
  a row's sum over the tokens: by tiles of 64, then lanes and partial results:                L / 64 + 40
  its rescaling, 1 / sum and the product with it:                                             23
  the sums over rows (a wave's share of 32), lanes, blocks and heads:                         R / 32 + H + 16
"""

import numpy as np

from oracle import attention as A


def largest_score(q, rows, w_uk, scale):
    """The largest score in size, times log2(e)."""
    q, rows, w_uk = (np.asarray(v, np.float64) for v in (q, rows, w_uk))
    Dn, Dc = w_uk.shape[1:]
    most = 0.0
    for h in range(q.shape[1]):
        s = (q[:, h, :Dn] @ w_uk[h]) @ rows[:, :Dc].T + q[:, h, Dn:] @ rows[:, Dc:].T
        most = max(most, np.abs(s).max(initial=0.0))
    return scale * most / np.log(2.0)


def total_tolerance(M, tokens, rows, heads):
    return A.SINGLE * (1.4 * (2 * M + 15) + 2.8 * (M + 7) + 6 + tokens / 64 + 40 + 23 + rows / 32 + heads + 16)


def check_added(got, q, rows, w_uk, scale, seen=None):
    """``got [L]``: what ``q [n, H, .]`` added to sums of zero over the tokens ``rows``, row i seeing the first seen[i]."""
    got, (n, H), L = np.asarray(got, np.float64), q.shape[:2], len(rows)
    want, bound = A.token_weights(q, rows, w_uk, scale, seen)
    off = np.abs(got - want)
    assert (off <= bound + A.SINGLE * want).all(), ("token", (off - bound).max())
    assert np.linalg.norm(off) <= 8 * A.HALF * np.linalg.norm(want), ("norm", np.linalg.norm(off) / np.linalg.norm(want))
    pairs = H * (n if seen is None else int((np.asarray(seen) > 0).sum())) if L else 0
    tol = total_tolerance(largest_score(q, rows, w_uk, scale), L, n, H)
    assert abs(got.sum() - pairs) <= tol * pairs, ("total", got.sum(), pairs, tol)
