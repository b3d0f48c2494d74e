"""Latent attention against the float64 oracle: cache writes, the absorbed form (single tokens, with and without a
shared prefix) and the expanded form (ragged chunks). Every page is NaN but for the tokens that are there, table
entries beyond a sequence's pages are no page ids, and each value is held to the bound that the oracle derives."""

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


class Cache:
    """A paged cache holding the rows of ``lens`` sequences (and of a shared prefix) at scattered pages."""

    def __init__(self, torch, g, H, Dc, Dr, Dn, Dv, page, lens, prefix=0, spare=2, size=1.0):
        from paper_2609_18063_amd import binding as B
        self.B, self.torch = B, torch
        self.H, self.Dc, self.Dr, self.Dn, self.Dv, self.page, self.lens = H, Dc, Dr, Dn, Dv, page, lens
        self.scale = 1 / np.sqrt(Dn + Dr)
        self.spec = B.make_latent_spec(H, Dc, Dr, Dn, Dv, page, self.scale)
        self.w = (g.standard_normal((H, Dn + Dv, Dc)) / np.sqrt(Dc)).astype(np.float16)
        self.rows = [(g.standard_normal((n, Dc + Dr)) * size).astype(np.float16) for n in lens]
        self.prefix_rows = g.standard_normal((prefix, Dc + Dr)).astype(np.float16)
        per = [-(-n // page) for n in lens]
        n_pages = sum(per) + -(-prefix // page) + spare
        order = g.permutation(n_pages).astype(np.int32)
        pages = np.full((n_pages, page, Dc + Dr), np.nan, np.float16)
        table = np.full((len(lens) + 1, max(per) + 2), (1 << 30) + 5, np.int32)
        table[1::2] = -9
        at = 0
        for b, rows in enumerate(self.rows + [self.prefix_rows]):
            k = -(-len(rows) // page)
            ids = order[at:at + k]
            at += k
            for j, i in enumerate(ids):
                part = rows[j * page:(j + 1) * page]
                pages[i, :len(part)] = part
            if b < len(lens):
                table[b, :k] = ids
            else:
                self.prefix_ids = torch.from_numpy(ids.copy()).cuda()
        self.table_np = table
        self.pages, self.table = torch.from_numpy(pages).cuda(), torch.from_numpy(table).cuda()
        self.cache = B.latent_cache(self.pages, self.table)
        self.wt = torch.from_numpy(self.w).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def workspace(self, n):
        return self.torch.full((n,), 255, dtype=self.torch.uint8, device="cuda")

    def decode(self, q, lens=None, most=None, prefix=0, out=None, ws=None):
        torch = self.torch
        lens = self.lens[:len(q)] if lens is None else lens
        most = max(list(lens) + [0]) if most is None else most
        out = torch.full((len(q), self.H, self.Dv), 7.0, dtype=torch.float16, device="cuda") if out is None else out
        if ws is None:
            ws = self.workspace(self.B.latent_decode_workspace_bytes(self.spec, len(q), most, prefix))
        self.B.latent_decode(self.spec, self.cache, self.wt, torch.from_numpy(q).cuda(),
                             torch.tensor(lens, dtype=torch.int32, device="cuda"), most, out, self.status, ws,
                             prefix=self.prefix_ids if prefix else None, prefix_len=prefix)
        return out.cpu().numpy()

    def prefill(self, q, counts, spare_q=0, spare_kv=0, max_q=None):
        torch = self.torch
        qs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        ks = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int32)
        T, kv = qs[-1] + spare_q, int(ks[-1] + spare_kv)
        qt = torch.full((int(T), self.H, self.Dn + self.Dr), float("nan"), dtype=torch.float16, device="cuda")
        qt[:qs[-1]] = torch.from_numpy(q).cuda()
        out = torch.full((int(T), self.H, self.Dv), 7.0, dtype=torch.float16, device="cuda")
        ws = self.workspace(self.B.latent_prefill_workspace_bytes(self.spec, len(counts), kv))
        self.B.latent_prefill(self.spec, self.cache, self.wt, qt, torch.from_numpy(qs).cuda(), torch.from_numpy(ks).cuda(),
                              kv, int(max(counts)) if max_q is None else max_q, out, self.status, ws)
        got = out.cpu().numpy()
        assert (got[qs[-1]:] == 7).all()
        return got[:qs[-1]]

    def check(self, got, q, b, rows, seen=None):
        """got, q: [n, H, .] of sequence b over the rows."""
        worst = 0.0
        for h in range(self.H):
            want, bound = A.attend(q[:, h], rows, self.w[h, :self.Dn], self.w[h, self.Dn:], self.scale, seen)
            off = np.abs(got[:, h].astype(np.float64) - want)
            assert np.isfinite(got[:, h]).all() and (off <= bound).all(), (b, h, off.max(), (off - bound).max())
            # the bound takes every rounding at its largest and with one sign; they are a dozen independent
            # ones a value, so that in the norm they stay within a few halves of a step
            norm = np.linalg.norm(want)
            if norm:
                worst = max(worst, np.linalg.norm(off) / norm)
        assert worst <= 8 * A.HALF, (b, worst)


def _queries(g, n, c, size=1.5):
    return (g.standard_normal((n, c.H, c.Dn + c.Dr)) * size).astype(np.float16)


W, S = (512, 64, 128, 128), (128, 32, 64, 64)
DECODE = [
    (1, *S, 16, [1]), (1, *S, 16, [0]), (3, *S, 16, [15, 16, 17]), (16, *S, 32, [63, 64, 65, 0]), (17, *S, 64, [1, 300, 5]),
    (33, *S, 16, [129, 64]), (64, *S, 128, [1000]), (128, *S, 1024, [70, 2000]),
    (5, 256, 32, 64, 128, 32, [200, 33]), (20, 256, 64, 128, 64, 64, [500, 1, 0, 77]), (40, 256, 64, 64, 64, 16, [130]),
    (1, *W, 64, [700]), (16, *W, 16, [31, 1500]), (32, *W, 64, [0, 64, 2049, 3]), (33, *W, 32, [90]), (128, *W, 64, [1, 400]),
    (8, 512, 32, 64, 64, 256, [5000, 100]), (2, *S, 16, [7] * 70)]


@pytest.mark.parametrize("H,Dc,Dr,Dn,Dv,page,lens", DECODE)
def test_decode(torch_cuda, H, Dc, Dr, Dn, Dv, page, lens):
    g = np.random.default_rng(sum(lens) + H)
    c = Cache(torch_cuda, g, H, Dc, Dr, Dn, Dv, page, lens)
    q = _queries(g, len(lens), c)
    got = c.decode(q)
    assert int(c.status) == 0
    for b, rows in enumerate(c.rows):
        c.check(got[b:b + 1], q[b:b + 1], b, rows)
    again = c.decode(q, most=max(lens) + 1000)           # another bound, another cut of the work
    for b, rows in enumerate(c.rows):
        c.check(again[b:b + 1], q[b:b + 1], b, rows)


@pytest.mark.parametrize("H,dims,page,lens,prefix", [
    (1, S, 16, [1], 1), (3, S, 16, [0, 5, 100], 17), (8, S, 32, [40] * 9, 500), (20, S, 16, [0] * 30, 64), (16, W, 64, [10, 300, 0], 1000),
    (32, W, 32, [65, 64], 129), (64, W, 64, [100, 7, 33], 2000), (128, (256, 64, 64, 64), 16, [5, 5, 5, 5, 5, 5, 5], 333)])
def test_decode_shared_prefix(torch_cuda, H, dims, page, lens, prefix):
    g = np.random.default_rng(prefix)
    c = Cache(torch_cuda, g, H, *dims, page, lens, prefix=prefix)
    q = _queries(g, len(lens), c)
    got = c.decode(q, prefix=prefix)
    assert int(c.status) == 0
    for b, rows in enumerate(c.rows):
        c.check(got[b:b + 1], q[b:b + 1], b, np.concatenate([c.prefix_rows, rows]))


def test_decode_long_rows_far_scores(torch_cuda):
    """Scores of a wide range, the largest late: every earlier sum is rescaled."""
    g = np.random.default_rng(11)
    c = Cache(torch_cuda, g, 4, *S, 16, [900])
    c.rows[0][:, :] *= np.linspace(0.1, 3, 900)[:, None].astype(np.float16)
    flat = c.pages.view(-1, 160)
    idx = (c.table_np[0, np.arange(900) // 16].astype(np.int64) * 16 + np.arange(900) % 16)
    flat[torch_cuda.from_numpy(idx).cuda()] = torch_cuda.from_numpy(c.rows[0]).cuda()
    q = _queries(g, 1, c, 3.0)
    got = c.decode(q)
    for h in range(4):
        want, bound = A.attend(q[:, h], c.rows[0], c.w[h, :64], c.w[h, 64:], c.scale)
        assert (np.abs(got[:, h] - want) <= bound).all()


def test_decode_lengths_and_pages_out_of_range(torch_cuda):
    g = np.random.default_rng(12)
    B = __import__("paper_2609_18063_amd.binding", fromlist=["x"])
    c = Cache(torch_cuda, g, 6, *S, 16, [50, 40, 30])
    q = _queries(g, 3, c)
    got = c.decode(q, lens=[50, -3, 99], most=50)         # 99 is taken as 50, which the table's own 30 tokens do not fill
    assert int(c.status) & B.MOE_STATUS_BAD_LENGTH
    c.check(got[:1], q[:1], 0, c.rows[0])
    assert not got[1].any()
    c.status.zero_()
    c.table[0, 1] = c.pages.shape[0]                      # tokens 16 .. 31 have no page
    got = c.decode(q)
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE
    c.check(got[:1], q[:1], 0, np.concatenate([c.rows[0][:16], c.rows[0][32:]]))
    c.check(got[1:2], q[1:2], 1, c.rows[1])
    c.status.zero_()
    c.table[0, :4] = -1
    got = c.decode(q)
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE and not got[0].any()
    got = c.prefill(q[:1].repeat(3, 0), [1, 1, 1])
    assert not got[0].any()
    c.check(got[1:2], q[:1], 1, c.rows[1])


PREFILL = [
    (1, S, 16, [1], [1]), (3, S, 16, [5], [5]), (2, S, 16, [64], [64]), (2, S, 64, [65], [1]), (4, S, 16, [130, 0, 3], [129, 0, 3]),
    (3, S, 32, [300, 77], [200, 77]), (5, S, 128, [1000, 20], [7, 1]), (2, (256, 64, 128, 64), 16, [190, 66], [66, 65]),
    (3, (256, 32, 64, 128), 64, [129], [128]), (2, W, 64, [257, 128], [257, 1]), (8, W, 16, [400], [131]), (1, (512, 64, 64, 128), 1024, [1500], [1100]),
    (7, (128, 64, 128, 128), 16, [3] * 40, [2] * 40)]


@pytest.mark.parametrize("H,dims,page,lens,counts", PREFILL)
def test_prefill(torch_cuda, H, dims, page, lens, counts):
    g = np.random.default_rng(sum(lens) + H)
    c = Cache(torch_cuda, g, H, *dims, page, lens)
    q = _queries(g, sum(counts), c)
    for kw in (dict(), dict(spare_q=5, spare_kv=70)):
        got = c.prefill(q, counts, **kw)
        assert int(c.status) == 0
        at = 0
        for b, n in enumerate(counts):
            if n:
                c.check(got[at:at + n], q[at:at + n], b, c.rows[b], np.arange(lens[b] - n, lens[b]) + 1)
            at += n


def test_prefill_is_decode(torch_cuda):
    """Both forms of one token agree within both bounds."""
    g = np.random.default_rng(13)
    c = Cache(torch_cuda, g, 16, *W, 64, [300, 1, 64])
    q = _queries(g, 3, c)
    a, b = c.decode(q), c.prefill(q, [1, 1, 1])
    assert np.linalg.norm(a.astype(np.float64) - b) <= 16 * A.HALF * np.linalg.norm(a.astype(np.float64))


def test_prefill_broken_lists(torch_cuda):
    """Lists that break the rules set the status; a chunk longer than its context starts with rows that see nothing."""
    g = np.random.default_rng(14)
    from paper_2609_18063_amd import binding as B
    c = Cache(torch_cuda, g, 3, *S, 16, [40, 9])
    q = _queries(g, 60, c)
    got = c.prefill(q[:57], [48, 9])
    assert int(c.status) == B.MOE_STATUS_BAD_LENGTH
    assert not got[:8].any()
    c.check(got[8:48], q[8:48], 0, c.rows[0], np.arange(40) + 1)
    c.check(got[48:57], q[48:57], 1, c.rows[1], np.arange(9) + 1)


def test_prefill_lost_pages(torch_cuda):
    g = np.random.default_rng(15)
    from paper_2609_18063_amd import binding as B
    c = Cache(torch_cuda, g, 3, *S, 16, [100, 50])
    q = _queries(g, 130, c)
    c.table[0, 2] = -1                                    # tokens 32 .. 47
    got = c.prefill(q, [100, 30])
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE
    kept = np.r_[0:32, 48:100]
    c.check(got[kept], q[kept], 0, c.rows[0][kept], np.arange(84) + 1)
    c.check(got[100:], q[100:], 1, c.rows[1], np.arange(20, 50) + 1)


@pytest.mark.parametrize("H,dims,page,T", [(1, S, 16, 1), (5, S, 16, 40), (32, W, 64, 7), (20, (256, 64, 128, 64), 128, 300), (0, W, 16, 9)])
def test_append(torch_cuda, H, dims, page, T):
    """Values, what is left alone (padding tokens, tokens out of range, other rows), and q in place."""
    torch, g = torch_cuda, np.random.default_rng(T)
    from paper_2609_18063_amd import binding as B
    Dc, Dr, Dn, Dv = dims
    c = Cache(torch, g, max(H, 1), *dims, page, [T + 20, 33])
    before = c.pages.clone()
    rope = A.rope_table(T + 20, Dr)
    kv = g.standard_normal((T, Dc + Dr)).astype(np.float32)
    kv[0] *= 1e-4
    gamma = (1 + 0.1 * g.standard_normal(Dc)).astype(np.float16)
    seq, pos = np.zeros(T, np.int32), (np.arange(T) + 11).astype(np.int32)
    skip = []
    if T > 6:
        seq[1], seq[2], pos[3], pos[4] = -1, 99, T + 20, -1
        skip = [1, 2, 3, 4]
    dev = [torch.from_numpy(v).cuda() for v in (kv, gamma, rope, seq, pos)]
    qo = qn = None
    if H:
        qn = g.standard_normal((T, H, Dn + Dr)).astype(np.float16)
        qt = torch.from_numpy(qn).cuda()
        qo = torch.full_like(qt, 7.0)
    B.latent_append(c.spec, c.cache, *dev, c.status, q=qt if H else None, q_out=qo)
    assert int(c.status) == (B.MOE_STATUS_BAD_INDEX if skip else 0)
    keep = np.setdiff1d(np.arange(T), skip)
    want = A.cache_row(kv[keep], gamma, rope[pos[keep], :, 0], rope[pos[keep], :, 1])
    flat, was = c.pages.view(-1, Dc + Dr).cpu().numpy(), before.view(-1, Dc + Dr).cpu().numpy()
    at = c.table_np[0, pos[keep] // page].astype(np.int64) * page + pos[keep] % page
    # a rounding to fp16, and fp32 sums of Dc squares, a root and two products on the way
    bound = (A.HALF + (Dc + 8) * A.SINGLE) * np.abs(want) + 4 * A.SINGLE * np.abs(kv[keep]).max(-1, keepdims=True) + A.TINY
    assert (np.abs(flat[at] - want) <= bound).all()
    rest = np.setdiff1d(np.arange(len(flat)), at)
    assert np.array_equal(flat[rest], was[rest], equal_nan=True)
    if H:
        got, cs = qo.cpu().numpy(), rope[pos[keep]][:, None]
        assert np.array_equal(got[keep][..., :Dn], qn[keep][..., :Dn])
        turned = A.rotate(qn[keep][..., Dn:].astype(np.float64), cs[..., 0], cs[..., 1])
        assert (np.abs(got[keep][..., Dn:] - turned) <= A.HALF * np.abs(turned) + 8 * A.SINGLE * np.abs(qn).max() + A.TINY).all()
        assert (got[skip] == 7).all()
        B.latent_append(c.spec, c.cache, *dev, c.status, q=qt, q_out=qt)
        assert np.array_equal(qt.cpu().numpy()[keep], got[keep])


def test_graphs_of_both_forms(torch_cuda):
    """Captured calls on a side stream with changing lengths, replayed between eager calls: every replay equals the
    eager call on the same inputs."""
    torch, g = torch_cuda, np.random.default_rng(16)
    from paper_2609_18063_amd import binding as B
    c = Cache(torch, g, 16, 256, 64, 64, 64, 16, [300, 200, 100])
    q = torch.from_numpy(_queries(g, 3, c)).cuda()
    lens = torch.tensor([300, 200, 100], dtype=torch.int32, device="cuda")
    out = torch.empty(3, 16, 64, dtype=torch.float16, device="cuda")
    out2 = torch.empty_like(out)
    starts = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    kvs = torch.tensor([0, 300, 500, 600], dtype=torch.int32, device="cuda")
    ws = c.workspace(B.latent_decode_workspace_bytes(c.spec, 3, 300))
    ws2 = c.workspace(B.latent_prefill_workspace_bytes(c.spec, 3, 600))

    def call():
        B.latent_decode(c.spec, c.cache, c.wt, q, lens, 300, out, c.status, ws)
        B.latent_prefill(c.spec, c.cache, c.wt, q, starts, kvs, 600, 1, out2, c.status, ws2)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    for n in ([300, 200, 100], [1, 0, 64], [65, 200, 17], [300, 200, 100]):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        kvs.copy_(torch.tensor(np.concatenate([[0], np.cumsum(np.maximum(n, 1))]), dtype=torch.int32))
        q.copy_(torch.from_numpy(_queries(g, 3, c)))
        graph.replay()
        a, b = out.clone(), out2.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, out2), n
        assert int(c.status) == 0


@pytest.mark.parametrize("H,lens,prefix", [(4, [3, 0] * 35, 6000), (8, [0, 1, 33, 70] * 16, 6300), (2, [40], 6000)])
def test_decode_prefix_by_more_rows(torch_cuda, H, lens, prefix):
    """Few heads of many sequences over a prefix: rows of several sequences in a workgroup, 16, 32 and 64 of them."""
    test_decode_shared_prefix(torch_cuda, H, S, 16, lens, prefix)


@pytest.mark.parametrize("dims,H", [(S, 3), (W, 8), ((256, 32, 64, 128), 2)])
@pytest.mark.parametrize("what,part", [(np.nan, 0), (np.inf, 0), (-np.inf, 1), (np.nan, 1), (6e4, 0)])
def test_prefill_later_tokens_stay_out(torch_cuda, dims, H, what, part):
    """A token that is not finite, or whose values are beyond fp16, changes no row before it and no other sequence."""
    g = np.random.default_rng(17)
    lens, counts, bad = [300, 90], [120, 90], 250
    c = Cache(torch_cuda, g, H, *dims, 16, lens)
    q = _queries(g, sum(counts), c)
    clean = c.prefill(q, counts)
    row = int(c.table_np[0, bad // 16]) * 16 + bad % 16
    flat = c.pages.view(-1, dims[0] + dims[1])
    flat[row, dims[0] * part:dims[0] + dims[1] if part else dims[0]] = float(what)
    got = c.prefill(q, counts)
    seen = bad - (lens[0] - counts[0])                    # the first row that sees the token
    assert np.array_equal(got[:seen], clean[:seen]) and np.array_equal(got[counts[0]:], clean[counts[0]:])
    if np.isnan(what):
        assert np.isnan(got[seen:counts[0]]).all()


@pytest.mark.parametrize("H,dims,page,lens,counts", [(1, S, 64, [40000], [3]), (2, S, 16, [20001, 15000], [1, 40])])
def test_long_contexts(torch_cuda, H, dims, page, lens, counts):
    test_prefill(torch_cuda, H, dims, page, lens, counts)
    test_decode(torch_cuda, H, *dims, page, lens)


def test_cache_past_32_bits(torch_cuda):
    """Rows at byte and element offsets beyond 2^32 and 2^31: written, copied to another page and read by both forms."""
    torch, g = torch_cuda, np.random.default_rng(18)
    from paper_2609_18063_amd import binding as B
    c = Cache(torch, g, 3, *S, 1024, [90])
    n_pages, row = 14000, S[0] + S[1]
    big = torch.empty(n_pages, 1024, row, dtype=torch.float16, device="cuda")
    assert big.numel() > 1 << 31
    far = n_pages - 3
    table = torch.tensor([[far], [far + 1]], dtype=torch.int32, device="cuda")
    cache = B.latent_cache(big, table)
    kv = torch.from_numpy(g.standard_normal((90, row)).astype(np.float32)).cuda()
    rope = torch.zeros(90, S[1] // 2, 2, device="cuda")
    rope[..., 0] = 1
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    B.latent_append(c.spec, cache, kv, torch.ones(S[0], dtype=torch.float16, device="cuda"), rope, i32([0] * 90), i32(list(range(90))),
                    c.status)
    x = kv.cpu().numpy().astype(np.float64)
    want = np.concatenate([x[:, :S[0]] / np.sqrt((x[:, :S[0]] ** 2).mean(-1, keepdims=True) + 1e-6), x[:, S[0]:]], 1)
    rows = big[far, :90].cpu().numpy()
    assert (np.abs(rows - want) <= np.abs(want) * (A.HALF + 1e-5) + 1e-7).all()  # one rounding to fp16, fp32 before it
    B.page_copy(big[None], i32([[far, far + 1], [far, 5]]), c.status)
    for p in (far + 1, 5):
        assert np.array_equal(big[p, :90].cpu().numpy(), rows)
    c.cache, c.lens, c.rows = cache, [90, 90], [rows, rows]
    q = _queries(g, 2, c)
    for got in (c.decode(q), c.prefill(q, [1, 1])):
        for b in range(2):
            c.check(got[b:b + 1], q[b:b + 1], b, rows)
    assert int(c.status) == 0
