"""NaN in latent attention: a row that sees one is NaN, in both forms and however the context is cut among workgroups,
and no other row changes."""

import numpy as np
import pytest

from oracle import attention as A
from tests.test_gpu_latent import Cache, S, W, _queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _at(c, b, tok):
    """Token ``tok`` of sequence ``b`` in the pages, as a row of halves."""
    return c.pages.view(-1, c.Dc + c.Dr)[int(c.table_np[b, tok // c.page]) * c.page + tok % c.page]


def _heads_are_right(c, got, q, rows, heads):
    for h in heads:
        want, bound = A.attend(q[:, h], rows, c.w[h, :c.Dn], c.w[h, c.Dn:], c.scale)
        assert (np.abs(got[:, h].astype(np.float64) - want) <= bound).all(), h


@pytest.mark.parametrize("most", [700, 5000, 130000])
@pytest.mark.parametrize("dims,H,lens", [(S, 3, [700, 65, 33]), (W, 20, [1, 700, 40]), (S, 2, [64])])
def test_decode_nan_query(torch_cuda, dims, H, lens, most):
    """One element of one head's query: that head's output is NaN, the sequence's other heads stay right, and the
    other sequences stay as they are."""
    g = np.random.default_rng(21)
    c = Cache(torch_cuda, g, H, *dims, 16, lens)
    q = _queries(g, len(lens), c)
    clean = c.decode(q, most=most)
    for b in range(len(lens)):
        for e in (3, c.Dn + 5):                            # in q_n and in q_r
            p = q.copy()
            p[b, 1, e] = np.nan
            got = c.decode(p, most=most)
            assert np.isnan(got[b, 1]).all()
            rest = np.setdiff1d(np.arange(H), [1])
            _heads_are_right(c, got[b:b + 1], q[b:b + 1], c.rows[b], rest)
            others = np.setdiff1d(np.arange(len(lens)), [b])
            assert np.array_equal(got[others], clean[others])


@pytest.mark.parametrize("most", [None, 4000, 130000])
@pytest.mark.parametrize("dims,H,lens", [(S, 3, [65]), (S, 3, [65, 300, 1]), (W, 32, [65, 33]), (W, 5, [2000, 1, 7])])
def test_decode_nan_token(torch_cuda, dims, H, lens, most):
    """A token that is alone in its tile, first in a tile, or the first of all, as a latent and as a key."""
    g = np.random.default_rng(22)
    c = Cache(torch_cuda, g, H, *dims, 16, lens)
    q = _queries(g, len(lens), c)
    clean = c.decode(q, most=most)
    for tok in sorted({lens[0] - 1, (lens[0] - 1) // 32 * 32, 0}):
        for part in (slice(2, 3), slice(c.Dc + 1, c.Dc + 2)):
            row = _at(c, 0, tok)
            was = row.clone()
            row[part] = float("nan")
            got = c.decode(q, most=most)
            row.copy_(was)
            assert np.isnan(got[0]).all(), (tok, part)
            assert np.array_equal(got[1:], clean[1:])


@pytest.mark.parametrize("dims,H,prefix", [(S, 3, 129), (W, 16, 1000)])
def test_decode_nan_in_a_shared_prefix(torch_cuda, dims, H, prefix):
    g = np.random.default_rng(23)
    lens = [65, 0, 5]
    c = Cache(torch_cuda, g, H, *dims, 16, lens, prefix=prefix)
    q = _queries(g, 3, c)
    p = q.copy()
    p[1, 2, 0] = np.nan                                    # (rows of several sequences share a workgroup)
    got = c.decode(p, prefix=prefix)
    assert np.isnan(got[1, 2]).all()
    for b in range(3):
        heads = np.setdiff1d(np.arange(H), [2]) if b == 1 else np.arange(H)
        _heads_are_right(c, got[b:b + 1], q[b:b + 1], np.concatenate([c.prefix_rows, c.rows[b]]), heads)
    last = c.pages[int(c.prefix_ids[(prefix - 1) // 16]), (prefix - 1) % 16]
    last[0] = float("nan")
    assert np.isnan(c.decode(q, prefix=prefix)).all()


@pytest.mark.parametrize("dims,H", [(S, 3), (W, 2)])
def test_prefill_nan_in_cut_contexts(torch_cuda, dims, H):
    """Contexts cut into parts: the first token that a row sees in its part (128: the first row block has four tiles in
    two parts), one further on, and a query."""
    g = np.random.default_rng(24)
    lens = counts = [2100, 90]
    assert sum(lens) // (len(lens) * 512) >= 2             # (from there on contexts are cut)
    c = Cache(torch_cuda, g, H, *dims, 16, lens)
    q = _queries(g, sum(counts), c)
    clean = c.prefill(q, counts)
    for bad in (128, 1000):
        row = _at(c, 0, bad)
        was = row.clone()
        row[:c.Dc] = float("nan")
        got = c.prefill(q, counts)
        row.copy_(was)
        assert np.array_equal(got[:bad], clean[:bad]) and np.array_equal(got[counts[0]:], clean[counts[0]:])
        assert np.isnan(got[bad:counts[0]]).all()
    for i in (0, 130, 2099, 2150):
        p = q.copy()
        p[i, 1, 0] = np.nan
        got = c.prefill(p, counts)
        assert np.isnan(got[i, 1]).all()
        same = np.ones(got.shape[:2], bool)
        same[i, 1] = False
        assert np.array_equal(got[same], clean[same])
