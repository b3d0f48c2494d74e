"""The checks of the 4-bit cache's sums tell mistakes of a launch from its roundings: mistakes planted in the oracle's own
weights, at the sizes of the GPU tests."""

import numpy as np
import pytest

from oracle import attention as A
from tests.latent4_sums import check_added


def _case(H, L, n, seed, dims=(128, 32, 64)):
    g, (Dc, Dr, Dn) = np.random.default_rng(seed), dims
    rows = A.row_values(*A.quantize_row(g.standard_normal((L, Dc + Dr)), Dc), Dc)
    w = (g.standard_normal((H, Dn, Dc)) / np.sqrt(Dc)).astype(np.float16)
    q = (g.standard_normal((n, H, Dn + Dr)) * 1.5).astype(np.float16)
    return q, rows, w, 1 / np.sqrt(Dn + Dr)


def _rounded(q, rows, w, scale, seen=None):
    """The weights with the roundings of a launch: operands to fp16, sums to fp32."""
    Dc, Dn = w.shape[2], w.shape[1]
    total = np.zeros(len(rows), np.float32)
    half = lambda x: np.asarray(x, np.float64).astype(np.float16).astype(np.float64)  # noqa: E731
    for h in range(q.shape[1]):
        s = scale * (half(q[:, h, :Dn].astype(np.float64) @ w[h]) @ half(rows[:, :Dc]).T + q[:, h, Dn:].astype(np.float64) @ half(rows[:, Dc:]).T)
        if seen is not None:
            s = np.where(np.arange(len(rows)) >= np.asarray(seen)[:, None], -np.inf, s)
        p = np.exp(s - s.max(-1, keepdims=True))
        for row in p / p.sum(-1, keepdims=True):
            total += row.astype(np.float32)
    return total


SHAPES = [(128, 400, 1, (128, 32, 64)), (40, 130, 1, (512, 64, 128)), (128, 500, 1, (128, 32, 64)), (33, 64, 1, (256, 32, 64)), (20, 300, 7, (128, 32, 64))]


@pytest.mark.parametrize("H,L,n,dims", SHAPES)
def test_roundings_pass(H, L, n, dims):
    q, rows, w, scale = _case(H, L, n, H + L, dims)
    seen = None if n == 1 else np.arange(L - n, L) + 1
    check_added(_rounded(q, rows, w, scale, seen), q, rows, w, scale, seen)


@pytest.mark.parametrize("H,L,n,dims", SHAPES)
def test_mistakes_fail(H, L, n, dims):
    """A head left out or taken twice, a block of 16 heads left out, a row left out, sums that are a thousandth too
    large, one token's neighbours exchanged by blocks of 16."""
    q, rows, w, scale = _case(H, L, n, H + L, dims)
    seen = np.arange(L - n, L) + 1
    whole = A.token_weights(q, rows, w, scale, seen)[0]
    heads = lambda a, b: A.token_weights(q[:, a:b], rows, w[a:b], scale, seen)[0]  # noqa: E731
    wrong = [whole - heads(0, 1), whole - heads(H - 1, H), whole + heads(H // 2, H // 2 + 1), whole - heads(H - 16, H), whole * 1.001,
             np.roll(whole, 16)]
    if n > 1:
        wrong.append(whole - A.token_weights(q[-1:], rows, w, scale, seen[-1:])[0])
    for got in wrong:
        with pytest.raises(AssertionError):
            check_added(got, q, rows, w, scale, seen)
