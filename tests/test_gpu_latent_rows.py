"""What else of a latent attention row's result may depend on: not on its neighbours' scores, not on how far its weights
lie apart; weights of the model that are not finite show."""

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


def _place(c, torch, b, rows):
    """The rows of sequence ``b``, into its pages."""
    c.rows[b] = rows
    i = np.arange(len(rows))
    at = c.table_np[b, i // c.page].astype(np.int64) * c.page + i % c.page
    c.pages.view(-1, c.Dc + c.Dr)[torch.from_numpy(at).cuda()] = torch.from_numpy(rows).cuda()


@pytest.mark.parametrize("dims,H,lens", [(S, 5, [700, 65, 33]), (W, 32, [400, 40])])
def test_decode_rows_for_themselves(torch_cuda, dims, H, lens):
    """Head 1's scores rise a hundredfold, or are infinite: the other heads' bits stay."""
    g = np.random.default_rng(51)
    c = Cache(torch_cuda, g, H, *dims, 16, lens)
    q = _queries(g, len(lens), c)
    clean = c.decode(q)
    rest = np.setdiff1d(np.arange(H), [1])
    for what in (100, np.inf):
        p = q.copy()
        p[:, 1] *= np.float16(what)
        assert np.array_equal(c.decode(p)[:, rest], clean[:, rest]), what


@pytest.mark.parametrize("dims,H,prefix", [(S, 5, 600), (W, 16, 300)])
def test_decode_sequences_for_themselves(torch_cuda, dims, H, prefix):
    """The same over a prefix that the batch shares, where rows of several sequences are in a workgroup."""
    g = np.random.default_rng(52)
    c = Cache(torch_cuda, g, H, *dims, 16, [65, 0, 200, 5], prefix=prefix)
    q = _queries(g, 4, c)
    clean = c.decode(q, prefix=prefix)
    p = q.copy()
    p[1] *= np.float16(100)
    rest = [0, 2, 3]
    assert np.array_equal(c.decode(p, prefix=prefix)[rest], clean[rest])


@pytest.mark.parametrize("dims,H,lens", [(S, 2, [300]), (W, 2, [300]), (S, 2, [2100])])
def test_prefill_rows_for_themselves(torch_cuda, dims, H, lens):
    """A token with far larger scores, or infinite ones, inside a wave's rows and tile: the rows before it keep their
    bits; and so do a row's neighbours where its query grows."""
    torch, g = torch_cuda, np.random.default_rng(53)
    c = Cache(torch, g, H, *dims, 16, lens)
    q = _queries(g, lens[0], c)
    q[:, :, c.Dn] = np.abs(q[:, :, c.Dn]) + np.float16(0.5)
    clean, original = c.prefill(q, lens), c.rows[0]
    for bad in (5, 40, 150, 250):
        rows = original.copy()
        for what in (200, np.inf):
            rows[bad, c.Dc] = what
            _place(c, torch, 0, rows)
            got = c.prefill(q, lens)
            assert np.array_equal(got[:bad], clean[:bad]), (bad, what)
            if np.isinf(what):
                assert np.isnan(got[bad:]).all()
    _place(c, torch, 0, original)
    for i in (7, 100, 299):
        p = q.copy()
        p[i] *= np.float16(100)
        rest = np.setdiff1d(np.arange(lens[0]), [i])
        assert np.array_equal(c.prefill(p, lens)[rest], clean[rest]), i


@pytest.mark.parametrize("dims", [S, W])
@pytest.mark.parametrize("nats", [0, 8, 12, 14, 16])
@pytest.mark.parametrize("form", ["decode", "prefill"])
def test_weights_far_below_the_largest(torch_cuda, dims, nats, form):
    """One token with a score ``nats`` above all others and a value of zero: the output is what the others add up to,
    at weights down to e^-16 of the largest (2^-23.1: held times 2^7 they are off by 2^-25 / 2^-16.1 = 4.2 A.HALF at
    most, alike for all of them, beside the roundings that 8 A.HALF are there for). All in one share of the work (a bound that large gives a workgroup 260
    tiles; contexts below 1,024 tokens are not cut)."""
    torch, g = torch_cuda, np.random.default_rng(54)
    n = 8000 if form == "decode" else 1000
    c = Cache(torch, g, 2, *dims, 64, [n])
    rows = np.zeros((n, c.Dc + c.Dr), np.float16)
    rows[1:, :c.Dc] = 1 + 0.25 * g.standard_normal((n - 1, c.Dc))
    rows[0, c.Dc] = nats / (8 * c.scale)                   # (its latent stays 0)
    _place(c, torch, 0, rows)
    q = np.zeros((1, 2, c.Dn + c.Dr), np.float16)
    q[0, :, c.Dn] = 8
    got = c.decode(q, most=1 << 26) if form == "decode" else c.prefill(q, [1])
    assert int(c.status) == 0
    c.check(got, q, 0, rows)


@pytest.mark.parametrize("dims", [S, W])
def test_weights_that_are_not_finite(torch_cuda, dims):
    """A NaN or an infinity in one row of W_uv shows in that column of that head, in both forms, and nowhere else."""
    torch, g = torch_cuda, np.random.default_rng(55)
    c = Cache(torch, g, 3, *dims, 16, [200])
    q = _queries(g, 200, c)
    for what in (np.nan, np.inf, -np.inf):
        wt = c.wt.clone()
        wt[1, c.Dn + 5, 7] = float(what)
        keep, c.wt = c.wt, wt
        outs = [c.decode(q[-1:]), c.prefill(q, [200])]
        c.wt = keep
        seen = [np.array([200]), np.arange(200) + 1]
        for got, qs, s in zip(outs, (q[-1:], q), seen):
            assert not np.isfinite(got[:, 1, 5]).any(), what
            for h in range(3):
                cols = np.setdiff1d(np.arange(c.Dv), [5]) if h == 1 else np.arange(c.Dv)
                want, bound = A.attend(qs[:, h], c.rows[0], c.w[h, :c.Dn], c.w[h, c.Dn:], c.scale, s)
                assert (np.abs(got[:, h].astype(np.float64) - want) <= bound)[:, cols].all(), (what, h)
