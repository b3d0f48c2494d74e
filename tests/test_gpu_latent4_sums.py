"""The 4-bit cache's sums of attention weights: what a call adds, token by token, in the norm and in total, over the forms
that heads, rows and lengths select; and rows that no output is formed of."""

import numpy as np
import pytest

from oracle import attention as A
from tests.latent4_sums import check_added
from tests.test_gpu_latent4 import M, PREFILL, S, W, Cache4, _queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _check(c, now, b, q, seen=None):
    """Row b of sums that were zero."""
    n = c.lens[b]
    check_added(now[b, :n], q, c.rows[b], c.w[:, :c.Dn], c.scale, seen)
    assert not now[b, n:].any()


@pytest.mark.parametrize("H,dims,lens", [
    (1, S, [300, 1]), (5, M, [65, 200]), (16, W, [700]), (17, S, [500, 1, 64]), (20, M, [2000, 33]), (32, W, [130, 1500]), (33, S, [300, 0, 64]),
    (40, W, [130, 1]), (48, S, [777]), (64, S, [1000]), (64, (256, 64, 128, 64), [65, 700]), (65, M, [129, 5]), (96, S, [400, 17]),
    (128, S, [400, 500, 70]), (128, W, [300])])
def test_decode_adds(torch_cuda, H, dims, lens):
    """Under a bound that is the longest length, and under far ones."""
    torch, g = torch_cuda, np.random.default_rng(H + sum(lens))
    c = Cache4(torch, g, H, *dims, 32, lens)
    q = _queries(g, len(lens), c)
    for most in (max(lens), 20000, 1 << 20):
        sums = torch.zeros(len(lens), most, device="cuda")
        c.decode(q, most=most, sums=sums)
        assert int(c.status) == 0
        now = sums[:, :max(lens) + 100].cpu().numpy()
        assert not sums[:, max(lens) + 100:].any()
        for b in range(len(lens)):
            _check(c, now, b, q[b:b + 1])


@pytest.mark.parametrize("H,dims,page,lens", [(2, S, 16, [40000, 33000]), (128, S, 64, [9000]), (16, W, 64, [33500])])
def test_decode_adds_over_long_contexts(torch_cuda, H, dims, page, lens):
    torch, g = torch_cuda, np.random.default_rng(sum(lens))
    c = Cache4(torch, g, H, *dims, page, lens)
    q = _queries(g, len(lens), c)
    sums = torch.zeros(len(lens), max(lens), device="cuda")
    c.decode(q, sums=sums)
    for b in range(len(lens)):
        _check(c, sums.cpu().numpy(), b, q[b:b + 1])


@pytest.mark.parametrize("B,dims", [(2500, S), (4300, (128, 64, 128, 64))])
def test_decode_adds_of_many_sequences(torch_cuda, B, dims):
    torch, g = torch_cuda, np.random.default_rng(B)
    lens = [int(n) for n in g.integers(0, 4, B)]
    lens[3], lens[B // 2], lens[-1] = 200, 65, 17
    c = Cache4(torch, g, 3, *dims, 16, lens)
    q = _queries(g, B, c)
    sums = torch.zeros(B, 200, device="cuda")
    c.decode(q, sums=sums)
    now = sums.cpu().numpy()
    for b in range(B):
        if lens[b]:
            _check(c, now, b, q[b:b + 1])
        else:
            assert not now[b].any()


@pytest.mark.parametrize("H,dims,page,lens,counts", PREFILL + [(20, S, 16, [700, 300], [300, 280]), (33, M, 32, [600], [520]), (128, S, 16, [90], [40])])
def test_prefill_adds(torch_cuda, H, dims, page, lens, counts):
    torch, g = torch_cuda, np.random.default_rng(sum(lens) + H)
    c = Cache4(torch, g, H, *dims, page, lens)
    q = _queries(g, sum(counts), c)
    sums = torch.zeros(len(lens), max(lens) + 40, device="cuda")
    c.prefill(q, counts, spare_q=5, spare_kv=70, sums=sums)
    assert int(c.status) == 0
    now, at = sums.cpu().numpy(), 0
    for b, n in enumerate(counts):
        if n:
            _check(c, now, b, q[at:at + n], np.arange(lens[b] - n, lens[b]) + 1)
        else:
            assert not now[b].any()
        at += n


@pytest.mark.parametrize("counts,context,max_q,rows", [
    ([300, 30], 200, 100, 256), ([700, 30], 0, 257, 512), ([30, 300], 90, 1, 256), ([300, 30], 3000, 100, 256)])
def test_prefill_rows_beyond_the_longest_chunk(torch_cuda, counts, context, max_q, rows):
    """A chunk longer than max_q, which the status tells: the rows that no output is formed of add nothing. (The workspace
    is NaN before the call.)"""
    torch, g = torch_cuda, np.random.default_rng(max_q)
    lens = [n + context for n in counts]
    c = Cache4(torch, g, 5, *S, 16, lens)
    q = _queries(g, sum(counts), c)
    sums = torch.zeros(2, max(lens), device="cuda")
    got = c.prefill(q, counts, max_q=max_q, sums=sums)
    assert int(c.status) == c.B.MOE_STATUS_BAD_LENGTH
    now, at = sums.cpu().numpy(), 0
    assert np.isfinite(now).all()
    for b, n in enumerate(counts):
        k = min(n, rows)
        seen = np.arange(lens[b] - n, lens[b])[:k] + 1
        c.check(got[at:at + k], q[at:at + k], b, c.rows[b], seen)
        assert (got[at + k:at + n] == 7).all()
        _check(c, now, b, q[at:at + k], seen)
        at += n
