"""The 4-bit latent cache against the float64 oracle: its writes to the bit, rows read back, both forms of attention
over what the codes stand for, and the tokens' weights. Every page is NaN but for the tokens that are there, and table
entries beyond a sequence's pages are no page ids."""

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


class Cache4:
    """A paged 4-bit cache holding the quantized rows of ``lens`` sequences at scattered pages."""

    def __init__(self, torch, g, H, Dc, Dr, Dn, Dv, page, lens, spare=2, size=1.0, rows=None):
        from paper_2609_18063_amd import binding as B
        self.B, self.torch = B, torch
        self.H, self.Dc, self.Dr, self.Dn, self.Dv, self.page, self.lens = H, Dc, Dr, Dn, Dv, page, list(lens)
        self.scale = 1 / np.sqrt(Dn + Dr)
        self.spec = B.make_latent_spec(H, Dc, Dr, Dn, Dv, page, self.scale)
        self.w = (g.standard_normal((H, Dn + Dv, Dc)) / np.sqrt(Dc)).astype(np.float16)
        per = [-(-n // page) for n in lens]
        n_pages = sum(per) + spare
        order = g.permutation(n_pages).astype(np.int32)
        self.mem = A.Pages4(n_pages, page, Dc, Dr)
        table = np.full((len(lens) + 1, max(per) + 2), (1 << 30) + 5, np.int32)
        table[1::2] = -9
        at, self.rows = 0, []
        for b, n in enumerate(lens):
            table[b, :per[b]] = order[at:at + per[b]]
            at += per[b]
            raw = g.standard_normal((n, Dc + Dr)) * size if rows is None else rows[b]
            codes, s, z = A.quantize_row(raw, Dc)
            j = np.arange(n)
            self.mem.put(table[b, j // page], j % page, codes, s, z)
            self.rows.append(A.row_values(codes, s, z, Dc))
        self.spare_ids = order[at:]
        self.table_np = table
        self.pages, self.table = torch.from_numpy(self.mem.raw).cuda(), torch.from_numpy(table).cuda()
        self.cache = B.latent4_cache(self.spec, self.pages, self.table)
        self.wt = torch.from_numpy(self.w).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def workspace(self, n):
        return self.torch.full((max(n, 16),), 255, dtype=self.torch.uint8, device="cuda")

    def i32(self, v):
        return self.torch.tensor(np.asarray(v), dtype=self.torch.int32, device="cuda")

    def decode(self, q, lens=None, most=None, sums=None):
        torch = self.torch
        lens = self.lens[:len(q)] if lens is None else lens
        most = max(list(lens) + [0]) if most is None else most
        out = torch.full((len(q), self.H, self.Dv), 7.0, dtype=torch.float16, device="cuda")
        ws = self.workspace(self.B.latent4_decode_workspace_bytes(self.spec, len(q), most, sums is not None))
        self.B.latent4_decode(self.spec, self.cache, self.wt, torch.from_numpy(q).cuda(), self.i32(lens), most, out,
                              self.status, ws, sums=sums)
        return out.cpu().numpy()

    def prefill(self, q, counts, spare_q=0, spare_kv=0, max_q=None, sums=None):
        torch = self.torch
        qs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        ks = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int32)
        T, kv = int(qs[-1] + spare_q), int(ks[-1] + spare_kv)
        qt = torch.full((T, self.H, self.Dn + self.Dr), float("nan"), dtype=torch.float16, device="cuda")
        qt[:qs[-1]] = torch.from_numpy(q).cuda()
        out = torch.full((T, self.H, self.Dv), 7.0, dtype=torch.float16, device="cuda")
        ws = self.workspace(self.B.latent4_prefill_workspace_bytes(self.spec, T, len(counts), kv, sums is not None))
        self.B.latent4_prefill(self.spec, self.cache, self.wt, qt, self.i32(qs), self.i32(ks), kv,
                               int(max(counts)) if max_q is None else max_q, out, self.status, ws, sums=sums)
        got = out.cpu().numpy()
        assert (got[qs[-1]:] == 7).all()
        return got[:qs[-1]]

    def check(self, got, q, b, rows, seen=None):
        """got, q: [n, H, .] of sequence b over the rows."""
        worst = 0.0
        for h in range(self.H):
            want, bound = A.attend(q[:, h], rows, self.w[h, :self.Dn], self.w[h, self.Dn:], self.scale, seen, cached=A.HALF)
            off = np.abs(got[:, h].astype(np.float64) - want)
            assert np.isfinite(got[:, h]).all() and (off <= bound).all(), (b, h, off.max(), (off - bound).max())
            norm = np.linalg.norm(want)
            if norm:
                worst = max(worst, np.linalg.norm(off) / norm)
        # (in the norm the roundings, independent of each other, stay within a few halves of a step)
        assert worst <= 8 * A.HALF, (b, worst)

    def check_sums(self, got, was, q, rows, seen=None):
        """got, was: a sequence's row of sums after and before."""
        n = len(rows)
        want, bound = A.token_weights(q, rows, self.w[:, :self.Dn], self.scale, seen)
        off = np.abs(got[:n].astype(np.float64) - was[:n].astype(np.float64) - want)
        assert (off <= bound + A.SINGLE * np.abs(was[:n]) * 2 + A.SINGLE * want).all(), (off - bound).max()
        assert np.array_equal(got[n:], was[n:], equal_nan=True)


def _queries(g, n, c, size=1.5):
    return (g.standard_normal((n, c.H, c.Dn + c.Dr)) * size).astype(np.float16)


def _sums(torch, g, n, width):
    """Rows of sums as a view with gaps; what is there before counts."""
    wide = torch.from_numpy(g.random((n, width + 5)).astype(np.float32)).cuda()
    return wide, wide[:, :width]


W, S, M = (512, 64, 128, 128), (128, 32, 64, 64), (256, 32, 64, 128)
DECODE = [
    (1, *S, 16, [1]), (1, *S, 16, [0]), (3, *S, 16, [15, 16, 17]), (16, *S, 32, [63, 64, 65, 0]), (17, *S, 64, [1, 300, 5]),
    (33, *S, 16, [129, 64]), (64, *S, 128, [1000]), (128, *S, 1024, [70, 2000]),
    (5, *M, 32, [200, 33]), (20, 256, 64, 128, 64, 64, [500, 1, 0, 77]), (40, 256, 64, 64, 64, 16, [130]),
    (1, *W, 64, [700]), (16, *W, 16, [31, 1500]), (32, *W, 64, [0, 64, 2049, 3]), (33, *W, 32, [90]), (128, *W, 64, [1, 400]),
    (8, 512, 32, 64, 64, 256, [5000, 100]), (2, *S, 16, [7] * 70), (65, 512, 32, 64, 128, 16, [77, 1])]


@pytest.mark.parametrize("H,dims,page,T", [(1, S, 16, 1), (5, S, 16, 40), (32, W, 64, 7), (20, (256, 64, 128, 64), 128, 300), (0, W, 16, 9)])
def test_append_and_read(torch_cuda, H, dims, page, T):
    """Codes, steps and middles to the bit, what is left alone, q in place; the rows as they are read back."""
    torch, g = torch_cuda, np.random.default_rng(T)
    Dc, Dr, Dn, Dv = dims
    c = Cache4(torch, g, max(H, 1), *dims, page, [T + 20, 33])
    B = c.B
    rope = A.rope_table(T + 90, Dr)
    kv = g.standard_normal((T, Dc + Dr)).astype(np.float32)
    kv[0] *= 1e-4
    if T > 6:
        kv[5, Dc:] = 3.0e-7                              # steps below fp16's smallest
        kv[6, :] = 0.0
    gamma = (1 + 0.1 * g.standard_normal(Dc)).astype(np.float16)
    seq, slot = np.zeros(T, np.int32), (np.arange(T) + 11).astype(np.int32)
    pos = slot + 70                                      # (as after an eviction)
    skip = []
    if T > 6:
        seq[1], seq[2], pos[3], slot[4] = -1, 99, T + 90, -1
        skip = [1, 2, 3, 4]
    dev = [torch.from_numpy(v).cuda() for v in (kv, gamma, rope, seq, slot, pos)]
    qo = qt = None
    if H:
        qn = g.standard_normal((T, H, Dn + Dr)).astype(np.float16)
        qt = torch.from_numpy(qn).cuda()
        qo = torch.full_like(qt, 7.0)
    B.latent4_append(c.spec, c.cache, *dev, c.status, q=qt, q_out=qo)
    assert int(c.status) == (B.MOE_STATUS_BAD_INDEX if skip else 0)
    keep = np.setdiff1d(np.arange(T), skip)
    want = A.cache_row(kv[keep], gamma, rope[pos[keep], :, 0].astype(np.float64), rope[pos[keep], :, 1].astype(np.float64))
    codes, s, z = A.quantize_row(want, Dc)
    c.mem.put(c.table_np[0, slot[keep] // page], slot[keep] % page, codes, s, z)
    assert np.array_equal(c.pages.cpu().numpy(), c.mem.raw)
    # every group is within half a step, a rounding of its middle and one of its step (7.5 of them) of its values
    g_of = np.minimum(np.arange(Dc + Dr) // 64, Dc // 64)
    off = np.abs(A.row_values(codes, s, z, Dc) - want)
    S64, Z64 = s.astype(np.float64)[:, g_of], np.abs(z.astype(np.float64))[:, g_of]
    assert (off <= S64 * (0.5 + 8 * A.HALF) + A.HALF * Z64 + 16 * A.TINY).all()
    rows = torch.full((T + 3, Dc + Dr), 7.0, dtype=torch.float16, device="cuda")
    back_seq, back_slot = np.append(seq, [0, 0, -1]).astype(np.int32), np.append(slot, [11, 0, 0]).astype(np.int32)
    if T > 6:
        back_seq[3], back_slot[3] = 0, 1 << 20
    c.status.zero_()
    B.latent4_read(c.spec, c.cache, c.i32(back_seq), c.i32(back_slot), rows, c.status)
    got = rows.cpu().numpy()
    assert int(c.status) == (B.MOE_STATUS_BAD_INDEX if skip else 0)
    assert np.array_equal(got[keep], A.row_values(codes, s, z, Dc).astype(np.float16))
    assert (got[skip] == 7).all() and (got[T + 2] == 7).all() and np.array_equal(got[T], got[0])
    assert np.array_equal(got[T + 1], c.rows[0][0].astype(np.float16))
    if H:
        got, cs = qo.cpu().numpy(), rope[pos[keep]][:, None]
        assert np.array_equal(got[keep][..., :Dn], qn[keep][..., :Dn])
        turned = A.rotate(qn[keep][..., Dn:].astype(np.float64), cs[..., 0], cs[..., 1])
        assert (np.abs(got[keep][..., Dn:] - turned) <= A.HALF * np.abs(turned) + 8 * A.SINGLE * np.abs(qn).max() + A.TINY).all()
        assert (got[skip] == 7).all()
        B.latent4_append(c.spec, c.cache, *dev, c.status, q=qt, q_out=qt)
        assert np.array_equal(qt.cpu().numpy()[keep], got[keep])


def test_append_of_many_rows(torch_cuda):
    """To the bit also where s or z, rounded to fp16 by way of fp32, is not what one rounding makes of it."""
    torch, g = torch_cuda, np.random.default_rng(77)
    Dc, Dr, Dn, Dv = S
    T, page = 30000, 64
    c = Cache4(torch, g, 1, *S, page, [1], spare=0)
    raw = torch.zeros(-(-T // page), c.pages.shape[1], dtype=torch.uint8, device="cuda")
    mem = A.Pages4(raw.shape[0], page, Dc, Dr)
    table = c.i32(range(raw.shape[0]))[None]
    kv = g.standard_normal((T, Dc + Dr)).astype(np.float32)
    gamma, rope = np.ones(Dc, np.float16), np.zeros((T, Dr // 2, 2), np.float32)
    rope[..., 0] = 1
    place = np.arange(T)
    c.B.latent4_append(c.spec, c.B.latent4_cache(c.spec, raw, table), torch.from_numpy(kv).cuda(), torch.from_numpy(gamma).cuda(),
                       torch.from_numpy(rope).cuda(), c.i32([0] * T), c.i32(place), c.i32(place), c.status)
    want = A.cache_row(kv, gamma, rope[..., 0].astype(np.float64), rope[..., 1].astype(np.float64))
    codes, s, z = A.quantize_row(want, Dc)
    lo, hi = want[:, :64].min(-1), want[:, :64].max(-1)
    assert (((hi - lo) / 15).astype(np.float16) != s[:, 0]).any()
    mem.raw[:] = 0
    mem.put(place // page, place % page, codes, s, z)
    assert np.array_equal(raw.cpu().numpy(), mem.raw) and int(c.status) == 0


def test_append_values_that_are_not_finite(torch_cuda):
    """A NaN, an infinity, or a step or middle beyond fp16 makes NaN of its group (of all latents, where the norm sees
    it), and of no other row."""
    torch, g = torch_cuda, np.random.default_rng(2)
    c = Cache4(torch, g, 1, *S, 16, [40])
    kv = g.standard_normal((8, 160)).astype(np.float32)
    gamma = np.ones(128, np.float16)
    gamma[70] = 60000
    kv[1, 3], kv[2, 130], kv[3, 140], kv[4, 128:] = np.nan, np.inf, 3e38, 1e5 * g.standard_normal(32)
    kv[5, 128:] = 70000.0 + 1e-3 * g.standard_normal(32)  # a small range around a middle that is beyond fp16
    kv[6, 70] = 1e6                                       # normed it is sqrt(128), times gamma beyond fp16
    rope = np.zeros((60, 16, 2), np.float32)
    rope[..., 0] = 1
    dev = [torch.from_numpy(v).cuda() for v in (kv, gamma, rope)]
    at = c.i32(np.arange(8) + 16)
    c.B.latent4_append(c.spec, c.cache, *dev, c.i32([0] * 8), at, at, c.status)
    with np.errstate(all="ignore"):
        want = A.cache_row(kv, gamma, rope[:8, :, 0], rope[:8, :, 1])
        codes, s, z = A.quantize_row(want, 128)
        want = A.row_values(codes, s, z, 128).astype(np.float16)
    rows = torch.zeros(8, 160, dtype=torch.float16, device="cuda")
    c.B.latent4_read(c.spec, c.cache, c.i32([0] * 8), at, rows, c.status)
    assert np.array_equal(rows.cpu().numpy(), want, equal_nan=True)
    nan = np.isnan(rows.cpu().numpy())
    assert nan[1, :128].all() and not nan[1, 128:].any() and nan[[2, 3, 5], 128:].all() and not nan[[0, 4, 7]].any()
    assert np.isinf(rows.cpu().numpy()[4, 128:]).any()   # (s and z of row 4 are in range: its values beyond it are infinite)
    assert nan[6, 64:128].all() and not nan[6, :64].any() and not nan[2:6, :64].any()
    assert int(c.status) == 0


@pytest.mark.parametrize("H,Dc,Dr,Dn,Dv,page,lens", DECODE)
def test_decode(torch_cuda, H, Dc, Dr, Dn, Dv, page, lens):
    torch, g = torch_cuda, np.random.default_rng(sum(lens) + H)
    c = Cache4(torch, g, H, Dc, Dr, Dn, Dv, page, lens)
    q = _queries(g, len(lens), c)
    got = c.decode(q)
    assert int(c.status) == 0
    for b, rows in enumerate(c.rows):
        c.check(got[b:b + 1], q[b:b + 1], b, rows)
    wide, sums = _sums(torch, g, len(lens), max(lens) + 1000)
    was = wide.cpu().numpy()
    again = c.decode(q, most=max(lens) + 1000, sums=sums)  # another bound, another cut of the work
    now = wide.cpu().numpy()
    for b, rows in enumerate(c.rows):
        c.check(again[b:b + 1], q[b:b + 1], b, rows)
        c.check_sums(now[b], was[b], q[b:b + 1], rows)
    wide.copy_(torch.from_numpy(was))
    assert np.array_equal(c.decode(q, most=max(lens) + 1000, sums=sums), again) and np.array_equal(wide.cpu().numpy(), now)


def test_decode_far_scores(torch_cuda):
    """Scores of a wide range, the largest late: every earlier sum is rescaled."""
    torch, g = torch_cuda, np.random.default_rng(11)
    rows = [g.standard_normal((900, 160)) * np.linspace(0.1, 3, 900)[:, None]]
    c = Cache4(torch, g, 4, *S, 16, [900], rows=rows)
    q = _queries(g, 1, c, 3.0)
    wide, sums = _sums(torch, g, 1, 900)
    was = wide.cpu().numpy()
    got = c.decode(q, sums=sums)
    for h in range(4):
        want, bound = A.attend(q[:, h], c.rows[0], c.w[h, :64], c.w[h, 64:], c.scale, cached=A.HALF)
        assert (np.abs(got[:, h] - want) <= bound).all()
    c.check_sums(wide.cpu().numpy()[0], was[0], q, c.rows[0])


def test_lengths_and_pages_out_of_range(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(12)
    c = Cache4(torch, g, 6, *S, 16, [50, 40, 30])
    B, q = c.B, _queries(g, 3, c)
    wide, sums = _sums(torch, g, 3, 60)
    was = wide.cpu().numpy()
    got = c.decode(q, lens=[50, -3, 99], most=50, sums=sums)  # 99 is taken as 50, which the table's own 30 tokens do not fill
    assert int(c.status) & B.MOE_STATUS_BAD_LENGTH
    c.check(got[:1], q[:1], 0, c.rows[0])
    c.check_sums(wide.cpu().numpy()[0], was[0], q[:1], c.rows[0])
    assert not got[1].any() and np.array_equal(wide.cpu().numpy()[1], was[1])
    c.status.zero_()
    wide.copy_(torch.from_numpy(was))
    c.table[0, 1] = c.pages.shape[0]                      # tokens 16 .. 31 have no page
    got = c.decode(q, sums=sums)
    now = wide.cpu().numpy()
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE
    kept = np.r_[0:16, 32:50]
    c.check(got[:1], q[:1], 0, c.rows[0][kept])
    c.check(got[1:2], q[1:2], 1, c.rows[1])
    want, bound = A.token_weights(q[:1], c.rows[0][kept], c.w[:, :64], c.scale)
    assert (np.abs(now[0][kept] - was[0][kept].astype(np.float64) - want) <= bound + 4 * A.SINGLE).all()
    assert np.array_equal(now[0][16:32], was[0][16:32])
    c.status.zero_()
    c.table[0, :4] = -1
    wide.copy_(torch.from_numpy(was))
    got = c.decode(q, sums=sums)
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE and not got[0].any() and np.array_equal(wide.cpu().numpy()[0], was[0])
    got = c.prefill(q[:1].repeat(3, 0), [1, 1, 1], sums=sums)
    assert not got[0].any() and np.array_equal(wide.cpu().numpy()[0], was[0])
    c.check(got[1:2], q[:1], 1, c.rows[1])


@pytest.mark.parametrize("dims,H,lens", [(S, 3, [65, 300, 1]), (W, 20, [700, 40]), (M, 64, [129, 64])])
@pytest.mark.parametrize("tok", [0, 64, -1])
def test_a_nan_group(torch_cuda, dims, H, lens, tok):
    """A token with a NaN group makes NaN of its sequence, in both forms and the sums, and of nothing else."""
    torch, g = torch_cuda, np.random.default_rng(22)
    c = Cache4(torch, g, H, *dims, 16, lens)
    tok = tok % lens[0]
    q = _queries(g, len(lens), c)
    _, sums = _sums(torch, g, len(lens), max(lens))
    was = sums.clone()
    clean, clean_sums = c.decode(q, sums=sums), sums.clone()
    clean2 = c.prefill(q, [1] * len(lens))
    for grp in (0, c.Dc // 64):
        raw = c.mem.raw.copy()
        page = c.table_np[0, tok // 16]
        raw[page, c.mem.steps:].view(np.float16).reshape(2, c.mem.G, 16)[1, grp, tok % 16] = np.nan
        c.pages.copy_(torch.from_numpy(raw))
        sums.copy_(was)
        got = c.decode(q, sums=sums)
        now = sums.cpu().numpy()
        assert np.isnan(got[0]).all() and np.array_equal(got[1:], clean[1:])
        assert np.isnan(now[0, :lens[0]]).all() and np.array_equal(now[1:], clean_sums.cpu().numpy()[1:])
        sums.copy_(was)
        got = c.prefill(q, [1] * len(lens), sums=sums)
        now = sums.cpu().numpy()
        assert np.isnan(got[0]).all() and np.array_equal(got[1:], clean2[1:])
        assert np.isnan(now[0, :lens[0]]).all() and np.isfinite(now[1:]).all()


def test_a_nan_query(torch_cuda):
    """One head's query: that head's output is NaN, and its sequence's sums; the other heads and sequences stay."""
    torch, g = torch_cuda, np.random.default_rng(23)
    c = Cache4(torch, g, 20, *S, 16, [300, 65])
    q = _queries(g, 2, c)
    _, sums = _sums(torch, g, 2, 300)
    was = sums.cpu().numpy()
    q[0, 7, 3] = np.nan
    got = c.decode(q, sums=sums)
    assert np.isnan(got[0, 7]).all() and np.isfinite(got[0, :7]).all() and np.isfinite(got[0, 8:]).all()
    assert np.isnan(sums[0].cpu().numpy()).all()
    c.check(got[1:], q[1:], 1, c.rows[1])
    c.check_sums(sums[1].cpu().numpy(), was[1], q[1:], c.rows[1])


PREFILL = [
    (1, S, 16, [1], [1]), (3, S, 16, [5], [5]), (2, S, 16, [64], [64]), (2, S, 64, [65], [1]), (4, S, 16, [130, 0, 3], [129, 0, 3]),
    (3, S, 32, [300, 77], [200, 77]), (5, S, 128, [1000, 20], [7, 1]), (2, (256, 64, 128, 64), 16, [190, 66], [66, 65]),
    (3, M, 64, [129], [128]), (2, W, 64, [257, 128], [257, 1]), (8, W, 16, [400], [131]), (1, (512, 64, 64, 128), 1024, [1500], [1100]),
    (7, (128, 64, 128, 128), 16, [3] * 40, [2] * 40), (2, S, 16, [5000], [3])]


@pytest.mark.parametrize("H,dims,page,lens,counts", PREFILL)
def test_prefill(torch_cuda, H, dims, page, lens, counts):
    torch, g = torch_cuda, np.random.default_rng(sum(lens) + H)
    c = Cache4(torch, g, H, *dims, page, lens)
    q = _queries(g, sum(counts), c)
    wide, sums = _sums(torch, g, len(lens), max(lens))
    was = wide.cpu().numpy()
    for kw in (dict(), dict(spare_q=5, spare_kv=70, sums=sums)):
        got = c.prefill(q, counts, **kw)
        assert int(c.status) == 0
        at, now = 0, wide.cpu().numpy()
        for b, n in enumerate(counts):
            seen = np.arange(lens[b] - n, lens[b]) + 1
            if n:
                c.check(got[at:at + n], q[at:at + n], b, c.rows[b], seen)
            if kw:
                c.check_sums(now[b], was[b], q[at:at + n], c.rows[b], seen)
            at += n
    wide.copy_(torch.from_numpy(was))
    assert np.array_equal(c.prefill(q, counts, spare_q=5, spare_kv=70, sums=sums), got) and np.array_equal(wide.cpu().numpy(), now)


def test_prefill_sums_of_fewer_tokens(torch_cuda):
    """Rows of sums shorter than a context: the tokens beyond them get none."""
    torch, g = torch_cuda, np.random.default_rng(5)
    c = Cache4(torch, g, 3, *S, 16, [200, 30])
    q = _queries(g, 60, c)
    wide, sums = _sums(torch, g, 2, 50)
    was = wide.cpu().numpy()
    c.prefill(q, [40, 20], sums=sums)
    now = wide.cpu().numpy()
    want, bound = A.token_weights(q[:40], c.rows[0], c.w[:, :64], c.scale, np.arange(160, 200) + 1)
    assert (np.abs(now[0, :50] - was[0, :50].astype(np.float64) - want[:50]) <= bound[:50] + 4 * A.SINGLE).all()
    assert np.array_equal(now[:, 50:], was[:, 50:])
    c.check_sums(now[1], was[1], q[40:], c.rows[1], np.arange(10, 30) + 1)


def test_prefill_lost_pages_and_broken_lists(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(15)
    c = Cache4(torch, g, 3, *S, 16, [100, 50])
    B, q = c.B, _queries(g, 130, c)
    c.table[0, 2] = -1                                    # tokens 32 .. 47
    _, sums = _sums(torch, g, 2, 100)
    was = sums.cpu().numpy()
    got = c.prefill(q, [100, 30], sums=sums)
    assert int(c.status) == B.MOE_STATUS_BAD_PAGE
    kept = np.r_[0:32, 48:100]
    now = sums.cpu().numpy()
    # (rows 32 .. 47 see the tokens before them only)
    seen = np.where(np.arange(100) < 32, np.arange(100) + 1, np.where(np.arange(100) < 48, 32, np.arange(100) - 15))
    c.check(got[:100], q[:100], 0, c.rows[0][kept], seen)
    want, bound = A.token_weights(q[:100], c.rows[0][kept], c.w[:, :64], c.scale, seen)
    assert (np.abs(now[0][kept] - was[0][kept].astype(np.float64) - want) <= bound + 4 * A.SINGLE).all()
    assert np.array_equal(now[0, 32:48], was[0, 32:48])
    c.check(got[100:], q[100:], 1, c.rows[1], np.arange(20, 50) + 1)
    c = Cache4(torch, g, 3, *S, 16, [40, 9])
    q = _queries(g, 60, c)
    got = c.prefill(q[:57], [48, 9], sums=_sums(torch, g, 2, 100)[1])
    assert int(c.status) == B.MOE_STATUS_BAD_LENGTH
    assert not got[:8].any()
    c.check(got[8:48], q[8:48], 0, c.rows[0], np.arange(40) + 1)
    c.check(got[48:57], q[48:57], 1, c.rows[1], np.arange(9) + 1)


def test_graphs_of_both_forms(torch_cuda):
    """Captured calls on a side stream with changing lengths, replayed between eager calls."""
    torch, g = torch_cuda, np.random.default_rng(16)
    c = Cache4(torch, g, 16, 256, 64, 64, 64, 16, [300, 200, 100])
    B = c.B
    q = torch.from_numpy(_queries(g, 3, c)).cuda()
    lens = c.i32([300, 200, 100])
    out = torch.empty(3, 16, 64, dtype=torch.float16, device="cuda")
    out2 = torch.empty_like(out)
    sums, sums2 = (torch.zeros(3, 300, device="cuda") for _ in range(2))
    starts, kvs = c.i32([0, 1, 2, 3]), c.i32([0, 300, 500, 600])
    ws = c.workspace(B.latent4_decode_workspace_bytes(c.spec, 3, 300, True))
    ws2 = c.workspace(B.latent4_prefill_workspace_bytes(c.spec, 3, 3, 600, True))

    def call():
        B.latent4_decode(c.spec, c.cache, c.wt, q, lens, 300, out, c.status, ws, sums=sums)
        B.latent4_prefill(c.spec, c.cache, c.wt, q, starts, kvs, 600, 1, out2, c.status, ws2, sums=sums2)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    for n in ([300, 200, 100], [1, 0, 64], [65, 200, 17], [300, 200, 100]):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        kvs.copy_(torch.tensor(np.concatenate([[0], np.cumsum(np.maximum(n, 1))]), dtype=torch.int32))
        q.copy_(torch.from_numpy(_queries(g, 3, c)))
        sums.zero_(), sums2.zero_()
        graph.replay()
        kept = [t.clone() for t in (out, out2, sums, sums2)]
        sums.zero_(), sums2.zero_()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, (out, out2, sums, sums2))), n
        assert int(c.status) == 0
        total = [16.0 if k else 0.0 for k in n]
        assert np.allclose(sums.sum(1).cpu().numpy(), total, rtol=1e-5)


@pytest.mark.parametrize("H,dims,lens", [
    (33, S, [300, 0, 64]), (64, S, [1000]), (128, S, [70, 500]), (65, M, [129, 5]), (64, (256, 64, 128, 64), [65, 700]), (40, W, [130, 1]),
    (128, W, [300])])
def test_decode_many_heads_and_a_far_bound(torch_cuda, H, dims, lens):
    """A bound on the lengths that is far above them: 64 query rows to a tile."""
    torch, g = torch_cuda, np.random.default_rng(H + sum(lens))
    c = Cache4(torch, g, H, *dims, 32, lens)
    q = _queries(g, len(lens), c)
    wide, sums = _sums(torch, g, len(lens), 1 << 20)
    was = wide[:, :2000].cpu().numpy()
    got = c.decode(q, most=1 << 20, sums=sums)
    assert int(c.status) == 0
    now = wide[:, :2000].cpu().numpy()
    for b, rows in enumerate(c.rows):
        c.check(got[b:b + 1], q[b:b + 1], b, rows)
        c.check_sums(now[b], was[b], q[b:b + 1], rows)


@pytest.mark.parametrize("H,dims,page,lens", [(2, S, 16, [40000, 33000]), (128, S, 64, [9000]), (16, W, 64, [33500])])
def test_long_contexts(torch_cuda, H, dims, page, lens):
    """Sums of several steps a workgroup. (Of the outputs' heads the oracle forms a few.)"""
    torch, g = torch_cuda, np.random.default_rng(sum(lens))
    c = Cache4(torch, g, H, *dims, page, lens)
    q = _queries(g, len(lens), c)
    wide, sums = _sums(torch, g, len(lens), max(lens))
    was = wide.cpu().numpy()
    got, now = c.decode(q, sums=sums), wide.cpu().numpy()
    assert int(c.status) == 0
    for b, rows in enumerate(c.rows):
        for h in {0, H // 2, H - 1}:
            want, bound = A.attend(q[b:b + 1, h], rows, c.w[h, :c.Dn], c.w[h, c.Dn:], c.scale, cached=A.HALF)
            assert (np.abs(got[b:b + 1, h].astype(np.float64) - want) <= bound).all(), (b, h)
        c.check_sums(now[b], was[b], q[b:b + 1], rows)


@pytest.mark.parametrize("B,dims", [(2500, S), (4300, (128, 64, 128, 64))])
def test_decode_of_many_sequences(torch_cuda, B, dims):
    """More sequences than a workgroup holds the lengths of; many of them empty."""
    torch, g = torch_cuda, np.random.default_rng(B)
    lens = [int(n) for n in g.integers(0, 4, B)]
    lens[3], lens[B // 2], lens[-1] = 200, 65, 17
    c = Cache4(torch, g, 1, *dims, 16, lens)
    q = _queries(g, B, c)
    wide, sums = _sums(torch, g, B, 200)
    was = wide.cpu().numpy()
    got, now = c.decode(q, sums=sums), wide.cpu().numpy()
    assert int(c.status) == 0
    assert not got[np.array(lens) == 0].any()
    for b in [0, 1, 2, 3, 4, B // 2 - 1, B // 2, B // 2 + 1, B - 2, B - 1] + list(range(7, B, 41)):
        if lens[b]:
            c.check(got[b:b + 1], q[b:b + 1], b, c.rows[b])
        c.check_sums(now[b], was[b], q[b:b + 1], c.rows[b])


def test_prefill_sums_of_a_nan_row(torch_cuda):
    """A NaN in one query row: NaN of that row, and of the sums of the tokens that it sees; those behind it stay."""
    torch, g = torch_cuda, np.random.default_rng(31)
    c = Cache4(torch, g, 2, *S, 16, [300, 20])
    q = _queries(g, 170, c)
    q[40, 1, 5] = np.nan                                  # sees tokens 0 .. 190
    _, sums = _sums(torch, g, 2, 300)
    was = sums.cpu().numpy()
    got, now = c.prefill(q, [150, 20], sums=sums), sums.cpu().numpy()
    assert int(c.status) == 0
    assert np.isnan(got[40, 1]).all() and np.isfinite(np.delete(got, 40, 0)).all()
    assert np.isnan(now[0, :191]).all()
    seen = np.arange(150, 300) + 1
    want, bound = A.token_weights(np.delete(q[:150], 40, 0), c.rows[0], c.w[:, :64], c.scale, np.delete(seen, 40))
    off = np.abs(now[0, 191:] - was[0, 191:].astype(np.float64) - want[191:])
    assert (off <= bound[191:] + 4 * A.SINGLE + A.SINGLE * want[191:]).all()
    c.check_sums(now[1], was[1], q[150:], c.rows[1], np.arange(20) + 1)


def test_cache_past_32_bits(torch_cuda):
    """Pages at byte offsets beyond 2^32: written, read back, moved and attended to by both forms."""
    torch, g = torch_cuda, np.random.default_rng(18)
    from paper_2609_18063_amd import binding as B
    H, n = 3, 90
    c = Cache4(torch, g, H, *S, 1024, [n])
    size = B.latent4_page_bytes(c.spec)
    n_pages = (1 << 32) // size + 60
    big = torch.empty(n_pages, size, dtype=torch.uint8, device="cuda")
    far = n_pages - 3
    table = torch.tensor([[far], [far + 1], [5]], dtype=torch.int32, device="cuda")
    cache = B.latent4_cache(c.spec, big, table)
    raw = g.standard_normal((n, S[0] + S[1])).astype(np.float32)
    rope = torch.zeros(n, S[1] // 2, 2, device="cuda")
    rope[..., 0] = 1
    place = c.i32(range(n))
    B.latent4_append(c.spec, cache, torch.from_numpy(raw).cuda(), torch.ones(S[0], dtype=torch.float16, device="cuda"), rope,
                     c.i32([0] * n), place, place, c.status)
    B.latent4_move(c.spec, big[None], table[:1].repeat(2, 1), place.view(1, 1, n).repeat(1, 2, 1), table[1:].contiguous(), c.status)
    x = raw.astype(np.float64)
    x[:, :S[0]] /= np.sqrt((x[:, :S[0]] ** 2).mean(-1, keepdims=True) + 1e-6)
    codes, s, z = A.quantize_row(x, S[0])
    rows = A.row_values(codes, s, z, S[0])
    for b in range(3):
        back = torch.empty(n, S[0] + S[1], dtype=torch.float16, device="cuda")
        B.latent4_read(c.spec, cache, c.i32([b] * n), place, back, c.status)
        assert (np.abs(back.cpu().numpy() - rows) <= np.abs(rows) * A.HALF + 2.0**-25).all()  # one rounding to fp16
    c.cache, c.lens, c.rows = cache, [n] * 3, [rows] * 3
    q = _queries(g, 3, c)
    was = np.zeros((3, n), np.float32)
    for call in (c.decode, lambda q, sums: c.prefill(q, [1, 1, 1], sums=sums)):
        sums = torch.zeros(3, n, device="cuda")
        got = call(q, sums=sums)
        for b in range(3):
            c.check(got[b:b + 1], q[b:b + 1], b, rows)
            c.check_sums(sums[b].cpu().numpy(), was[b], q[b:b + 1], rows)
    assert int(c.status) == 0


def test_calls_on_another_stream(torch_cuda):
    """The stream that a call names: what is ordered before it there is seen, what is ordered behind it sees it."""
    torch, g = torch_cuda, np.random.default_rng(4)
    c = Cache4(torch, g, 4, *M, 16, [150, 40])
    B, q = c.B, _queries(g, 2, c)
    qt = torch.from_numpy(q).cuda()
    late, out = torch.zeros_like(qt), torch.zeros(2, 4, M[3], dtype=torch.float16, device="cuda")
    sums = torch.zeros(2, 150, device="cuda")
    lens, ws = c.i32([150, 40]), c.workspace(B.latent4_decode_workspace_bytes(c.spec, 2, 150, True))
    keep, kept = torch.zeros(1, 2, 30, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, 150, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2000000)
        late.copy_(qt)
    B.latent4_decode(c.spec, c.cache, c.wt, late, lens, 150, out, c.status, ws, sums=sums, stream=side)
    B.evict_select(sums[None], lens, 30, 2, 5, keep, kept, c.status, stream=side)
    side.synchronize()
    for b in range(2):
        c.check(out[b:b + 1].cpu().numpy(), q[b:b + 1], b, c.rows[b])
        want = A.evict(sums[b].cpu().numpy(), c.lens[b], 30, 2, 5)
        assert keep[0, b].tolist() == want
        assert torch.equal(kept[0, b, :30], sums[b][torch.tensor(want, device="cuda")])
    assert int(c.status) == 0
