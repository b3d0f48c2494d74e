"""Page copies and table rewrites on the device: bit for bit what indexing gives, in several layers, with pages of a
few bytes and of many, and a pool's forks and compactions carried out on a cache."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


@pytest.mark.parametrize("layers,n_pages,halves,moves", [(1, 2, 8, 1), (3, 9, 24, 4), (2, 40, 16 * 160, 17), (5, 64, 64 * 576, 30), (2, 5, 8200, 2)])
def test_copies(torch_cuda, layers, n_pages, halves, moves):
    torch, g = torch_cuda, np.random.default_rng(halves)
    from paper_2609_18063_amd import binding as B
    wide = torch.from_numpy(g.integers(0, 1 << 15, (layers, n_pages + 3, halves)).astype(np.int16)).cuda()
    pages = wide[:, :n_pages]                              # layers further apart than their pages need
    order = g.permutation(n_pages)[:2 * moves].astype(np.int32).reshape(2, moves)
    want = wide.clone()
    want[:, order[1]] = want[:, order[0]]
    pairs = torch.from_numpy(np.ascontiguousarray(order.T)).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.page_copy(pages, pairs, status)
    assert torch.equal(wide, want) and int(status) == 0
    bad = torch.tensor([[0, n_pages], [-1, 0], [n_pages, 0], [0, -5]], dtype=torch.int32, device="cuda")
    B.page_copy(pages, bad, status)
    assert torch.equal(wide, want) and int(status) == B.MOE_STATUS_BAD_PAGE
    B.page_copy(pages, pairs[:0], status)


@pytest.mark.parametrize("n", [1, 255, 256, 1000])
def test_remap(torch_cuda, n):
    torch, g = torch_cuda, np.random.default_rng(n)
    from paper_2609_18063_amd import binding as B
    remap = torch.from_numpy(g.permutation(50).astype(np.int32)).cuda()
    table = torch.from_numpy(g.integers(-2, 50, n).astype(np.int32)).cuda()
    want = torch.where(table >= 0, remap[table.clamp_min(0).long()], table)
    out, status = torch.full_like(table, 7), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.page_remap(table, remap, out, status)
    assert torch.equal(out, want) and int(status) == 0
    table[0] = 50
    want[0] = 50
    B.page_remap(table, remap, table, status)              # in place; an id past the pages stays and is reported
    assert torch.equal(table, want) and int(status) == B.MOE_STATUS_BAD_PAGE


def test_pool_on_a_cache(torch_cuda):
    """Random forks, writes, frees and compactions: every sequence's tokens stay what was written."""
    torch, g = torch_cuda, np.random.default_rng(3)
    from paper_2609_18063_amd import binding as B
    L, N, P, R = 2, 60, 16, 8
    pool, pages = B.PagePool(N, P), torch.zeros(L, N, P, R, dtype=torch.float16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    seqs, clock = [], 0                                    # (pages, token stamps)
    for step in range(250):
        op = g.integers(6)
        if op <= 2 and pool.available() >= 4:
            if op == 2 and seqs:                           # fork a sequence at any of its tokens
                ids, text = seqs[g.integers(len(seqs))]
                n = int(g.integers(1, len(text) + 1))
                ids, pairs = pool.fork(ids, n)
                text = list(text[:n])
                if pairs:
                    B.page_copy(pages, torch.tensor(pairs, dtype=torch.int32, device="cuda"), status)
            else:
                ids, text = [], []
            for _ in range(int(g.integers(1, 40))):        # write on at its end
                if len(text) % P == 0:
                    if pool.available() == 0:
                        break
                    ids = ids + pool.alloc(1)
                clock += 1
                pages[:, ids[-1], len(text) % P] = clock
                text = text + [clock]
            if ids:
                seqs.append((ids, text))
        elif op == 3 and seqs:
            pool.free(seqs.pop(g.integers(len(seqs)))[0])
        elif op == 4 and step % 3 == 0:
            moves, remap = pool.compact()
            if len(moves):
                B.page_copy(pages, torch.from_numpy(moves.copy()).cuda(), status)
            table = torch.tensor([i for ids, _ in seqs for i in ids] or [-1], dtype=torch.int32, device="cuda")
            B.page_remap(table, torch.from_numpy(remap).cuda(), table, status)
            flat, at = table.tolist(), 0
            for k, (ids, text) in enumerate(seqs):
                seqs[k] = (flat[at:at + len(ids)], text)
                at += len(ids)
        host = pages.float().cpu().numpy() if step % 10 == 0 else None
        if host is not None:
            for ids, text in seqs:
                got = host[:, ids].reshape(L, -1, R)[:, :len(text)]
                assert np.array_equal(got, np.broadcast_to(np.float16(text).astype(np.float32)[None, :, None], got.shape))
    assert int(status) == 0
    pool.close()
