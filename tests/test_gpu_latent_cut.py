"""Latent attention where the work is cut: wide heads over contexts in parts, a lost page inside one, batches of more
sequences than a workgroup adds up at once, and weights far below a row's largest."""

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


@pytest.mark.parametrize("H,dims,page,lens,counts", [
    (8, W, 64, [1700], [5]), (3, W, 16, [5001, 40], [7, 3]), (2, (512, 32, 128, 64), 32, [9000, 1501, 2], [4, 130, 2]),
    (1, (128, 64, 128, 128), 16, [20001], [1]), (2, (256, 32, 128, 64), 128, [3000, 2999], [300, 1])])
def test_prefill_of_cut_contexts(torch_cuda, H, dims, page, lens, counts):
    assert sum(lens) // (len(lens) * 512) >= 2
    g = np.random.default_rng(sum(lens))
    c = Cache(torch_cuda, g, H, *dims, page, lens)
    q = _queries(g, sum(counts), c)
    got = c.prefill(q, counts)
    assert int(c.status) == 0
    at = 0
    for b, n in enumerate(counts):
        c.check(got[at:at + n], q[at:at + n], b, c.rows[b], np.arange(lens[b] - n, lens[b]) + 1)
        at += n


@pytest.mark.parametrize("dims", [W, (512, 32, 128, 64)])
def test_prefill_lost_page_in_a_part(torch_cuda, dims):
    from paper_2609_18063_amd import binding as B
    g = np.random.default_rng(31)
    c = Cache(torch_cuda, g, 3, *dims, 32, [3000])
    q = _queries(g, 9, c)
    c.table[0, 40] = -1                                    # tokens 1280 .. 1311
    got = c.prefill(q, [9])
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE
    c.check(got, q, 0, np.delete(c.rows[0], np.arange(1280, 1312), 0), np.arange(2991, 3000) - 32 + 1)


@pytest.mark.parametrize("H,B", [(2, 300), (1, 513)])
def test_decode_many_sequences(torch_cuda, H, B):
    g = np.random.default_rng(B)
    lens = [int(n) for n in g.integers(0, 70, B)]
    c = Cache(torch_cuda, g, H, *S, 16, lens)
    q = _queries(g, B, c)
    got = c.decode(q)
    assert int(c.status) == 0
    for b, rows in enumerate(c.rows):
        c.check(got[b:b + 1], q[b:b + 1], b, rows)
