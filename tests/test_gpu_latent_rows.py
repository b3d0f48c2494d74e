"""Latent attention's rows: weights of the model that are not finite show."""

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
