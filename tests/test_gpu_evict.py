"""Eviction against the oracle: which tokens stay, their sums, and their rows' bytes in the new pages."""

import numpy as np
import pytest

from oracle import attention as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _select(torch, sums, lens, budget, sinks, recent, inplace=False):
    from paper_2609_18063_amd import binding as B
    s = torch.from_numpy(sums).cuda()
    out = s if inplace else torch.full_like(s, 5.0)
    keep = torch.full((*sums.shape[:2], budget), 77, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.evict_select(s, torch.tensor(lens, dtype=torch.int32, device="cuda"), budget, sinks, recent, keep, out, status)
    if not inplace:
        assert np.array_equal(s.cpu().numpy(), sums, equal_nan=True)
    return keep.cpu().numpy(), out.cpu().numpy(), int(status)


def _expect(sums, lens, budget, sinks, recent):
    L, S, width = sums.shape
    keep, out = np.full((L, S, budget), -1, np.int32), np.zeros_like(sums)
    for layer in range(L):
        for b, n in enumerate(lens):
            ids = A.evict(sums[layer, b], n, budget, sinks, recent)
            keep[layer, b, :len(ids)] = ids
            out[layer, b, :len(ids)] = sums[layer, b, ids]
    return keep, out


def _make(g, kind, shape):
    v = np.exp(1.5 * g.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        v = np.floor(v * 2).astype(np.float32) / 2
    elif kind == "equal":
        v[:] = 3.0
    elif kind == "zero":
        v[:] = 0.0
        v.reshape(-1)[::7] = -0.0
    elif kind == "odd":
        flat = v.reshape(-1)
        flat[::5], flat[1::9], flat[3::11], flat[4::13] = np.nan, np.inf, -np.inf, -2.5
    elif kind == "near":                                  # keys that differ in their last bits only
        v = (np.float32(1000.0).view(np.int32) + g.integers(0, 5, shape)).astype(np.int32).view(np.float32)
    return v


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "zero", "odd", "near"])
@pytest.mark.parametrize("width,lens,budget,sinks,recent", [
    (1, [1], 1, 0, 0), (5, [5, 0, 3], 2, 1, 1), (7, [7, 6, 1], 3, 0, 0), (100, [100, 64, 20], 20, 4, 16), (100, [100], 100, 3, 3),
    (100, [100], 99, 0, 99), (1025, [1025, 1024, 300], 257, 0, 100), (4097, [4097, 4096, 1], 1000, 4, 0), (9001, [9001], 1, 0, 0),
    (9001, [8999], 8998, 2, 5)])
def test_select(torch_cuda, kind, width, lens, budget, sinks, recent):
    g = np.random.default_rng(width + budget)
    sums = _make(g, kind, (2, len(lens), width))
    want, moved = _expect(sums, lens, budget, sinks, recent)
    for inplace in (False, True):
        keep, out, status = _select(torch_cuda, sums, lens, budget, sinks, recent, inplace)
        assert status == 0
        assert np.array_equal(keep, want)
        assert np.array_equal(out, moved, equal_nan=True)


def test_select_long_row(torch_cuda):
    g = np.random.default_rng(4)
    sums = _make(g, "plain", (1, 2, 150_001))
    want, moved = _expect(sums, [150_001, 70_000], 40_000, 4, 1000)
    keep, out, _ = _select(torch_cuda, sums, [150_001, 70_000], 40_000, 4, 1000, True)
    assert np.array_equal(keep, want) and np.array_equal(out, moved)


def test_select_lengths_out_of_range(torch_cuda):
    from paper_2609_18063_amd import binding as B
    g = np.random.default_rng(3)
    sums = _make(g, "plain", (2, 3, 60))
    keep, out, status = _select(torch_cuda, sums, [-4, 61, 60], 10, 1, 2)
    assert status == B.MOE_STATUS_BAD_LENGTH
    want, moved = _expect(sums, [0, 60, 60], 10, 1, 2)
    assert np.array_equal(keep, want) and np.array_equal(out, moved)


@pytest.mark.parametrize("dims", [(512, 64), (512, 32), (256, 64), (256, 32), (128, 64), (128, 32)])
@pytest.mark.parametrize("page,lens,budget,layers", [(16, [100, 33, 0], 40, 3), (64, [200], 65, 1), (1024, [1500, 70], 130, 2), (32, [31, 32], 32, 2)])
def test_move(torch_cuda, dims, page, lens, budget, layers):
    """Kept rows' bytes in the new pages; every other byte stays. Two sequences may share the old pages."""
    torch, g = torch_cuda, np.random.default_rng(sum(lens))
    from paper_2609_18063_amd import binding as B
    Dc, Dr = dims
    spec = B.make_latent_spec(4, Dc, Dr, 64, 64, page, 0.1)
    S, per, need = len(lens), [-(-n // page) for n in lens], -(-budget // page)
    n_pages = sum(per) + need * S + 3
    order = g.permutation(n_pages).astype(np.int32)
    table = np.full((S, max(per) + 1), -1, np.int32)
    at = 0
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
    to = np.concatenate([order[at:at + need * S].reshape(S, need), np.full((S, 1), -7, np.int32)], 1)
    if S > 1:
        table[1, :per[1]] = table[0, :per[1]]             # a fork
    mem = [A.Pages4(n_pages, page, Dc, Dr) for _ in range(layers)]
    for m in mem:
        m.raw[:] = g.integers(0, 256, m.raw.shape)
    # (layers with a gap between them)
    wide = torch.from_numpy(np.stack([np.concatenate([m.raw.reshape(-1), np.zeros(64, np.uint8)]) for m in mem])).cuda()
    pages = wide[:, :-64].unflatten(1, (n_pages, -1))
    keep = np.full((layers, S, budget), -1, np.int32)
    for layer in range(layers):
        for b, n in enumerate(lens):
            k = min(n, budget)
            keep[layer, b, :k] = np.sort(g.permutation(n)[:k])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.latent4_move(spec, pages, torch.from_numpy(table).cuda(), torch.from_numpy(keep).cuda(), torch.from_numpy(to).cuda(), status)
    assert int(status) == 0
    for layer, m in enumerate(mem):
        was = m.raw.copy()
        for b in range(S):
            ids = keep[layer, b][keep[layer, b] >= 0]
            i = np.arange(len(ids))
            m.put(to[b, i // page], i % page, *m.get(table[b, ids // page], ids % page, was))
        assert np.array_equal(pages[layer].cpu().numpy(), m.raw)
    assert not wide[:, -64:].any()


def test_move_of_places_and_pages_out_of_range(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(8)
    from paper_2609_18063_amd import binding as B
    spec = B.make_latent_spec(4, 128, 32, 64, 64, 16, 0.1)
    m = A.Pages4(9, 16, 128, 32)
    m.raw[:] = g.integers(0, 256, m.raw.shape)
    pages = torch.from_numpy(m.raw).cuda()[None]
    for table, keep, to, status in (
            ([[0, 1, 2]], [3, 48, 49, 20], [[5]], B.MOE_STATUS_BAD_INDEX), ([[0, 9, 2]], [3, 16, 17, 40], [[5]], B.MOE_STATUS_BAD_PAGE),
            ([[0, 1, -1]], [3, 20, 32, 47], [[5]], B.MOE_STATUS_BAD_PAGE), ([[0, 1, 2]], [3, 20, 32, 47], [[9]], B.MOE_STATUS_BAD_PAGE),
            ([[0, 1, 2]], [3, 20, 32, 47], [[-1]], B.MOE_STATUS_BAD_PAGE)):
        got = pages.clone()
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        B.latent4_move(spec, got, i32(table), i32([[keep]]), i32(to), st)
        assert int(st) == status
        want = A.Pages4(9, 16, 128, 32)
        want.raw[:] = m.raw
        for i, slot in enumerate(keep):
            if slot < 48 and 0 <= table[0][slot // 16] < 9 and 0 <= to[0][0] < 9:
                want.put([to[0][0]], [i], *m.get([table[0][slot // 16]], [slot % 16]))
        assert np.array_equal(got[0].cpu().numpy(), want.raw)
