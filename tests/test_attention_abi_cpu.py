"""Argument checks of the attention block's calls, and the page pool against the oracle's, without a GPU (the
device addresses below are never dereferenced: a refused call enqueues nothing)."""

import ctypes

import numpy as np
import pytest

from oracle import attention as A


@pytest.fixture(scope="module")
def B():
    from paper_2609_18063_amd import binding
    binding.lib()
    return binding


P = [0x100000 * (i + 1) for i in range(16)]


def _linear(B, proj=None, out=64, inn=128, rank=4, x=P[4], xs=128, T=2, y=P[5], kind=0, ys=64, ws=P[6], wb=1 << 20,
            scale=2.0):
    proj = B.MoeProj(P[0], P[1], P[2], P[3]) if proj is None else proj
    return B.lib().moe_linear_int4_lora(ctypes.byref(proj) if proj else None, out, inn, rank, scale, x, xs, T, y, kind,
                                        ys, ws, wb, None)


def test_linear_refusals(B):
    assert _linear(B, T=0) == B.MOE_OK
    assert _linear(B, T=0, x=None, y=None, ws=None) == B.MOE_OK
    for bad in (dict(proj=False), dict(out=0), dict(inn=96), dict(inn=0), dict(inn=65536, xs=65536), dict(rank=65),
                dict(rank=0), dict(rank=-1), dict(T=-1), dict(kind=3), dict(xs=120), dict(xs=132), dict(ys=63),
                dict(x=None), dict(y=None), dict(ws=None), dict(scale=float("nan")), dict(proj=B.MoeProj(None, P[1], None, None)),
                dict(proj=B.MoeProj(P[0], None, None, None)), dict(out=(1 << 20) + 1, ys=1 << 21)):
        assert _linear(B, **bad) == B.MOE_EINVAL, bad
    for bad in (dict(x=P[4] + 8), dict(y=P[5] + 4), dict(ws=P[6] + 4), dict(proj=B.MoeProj(P[0] + 8, P[1], None, None)),
                dict(proj=B.MoeProj(P[0], P[1] + 4, None, None)), dict(proj=B.MoeProj(P[0], P[1], P[2] + 2, P[3]))):
        assert _linear(B, **bad) == B.MOE_EALIGN, bad
    need = B.linear_workspace_bytes(64, 128, 4, 2)
    assert need > 0 and _linear(B, wb=need - 1) == B.MOE_ENOMEM
    assert B.linear_workspace_bytes(64, 100, 4, 2) == 0 and B.linear_workspace_bytes(64, 128, 65, 2) == 0
    sizes = [B.linear_workspace_bytes(64, 4096, r, t) for r in (0, 64) for t in (1, 16, 17, 64, 65, 4000)]
    assert sizes[:6] == sorted(sizes[:6]) and sizes[6:] == sorted(sizes[6:]) and all(a <= b for a, b in zip(sizes, sizes[6:]))


def _spec(B, **kw):
    d = dict(heads=8, d_latent=128, d_rope=32, d_nope=64, d_v=64, page_tokens=16, scale=0.1)
    d.update(kw)
    return B.make_latent_spec(**d)


def test_latent_spec(B):
    assert B.latent_spec_check(_spec(B)) == B.MOE_OK
    for bad in (dict(heads=0), dict(heads=129), dict(d_latent=64), dict(d_latent=384), dict(d_latent=1024), dict(d_rope=16),
                dict(d_rope=128), dict(d_nope=32), dict(d_v=96), dict(page_tokens=8), dict(page_tokens=24),
                dict(page_tokens=2048), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert B.latent_spec_check(_spec(B, **bad)) == B.MOE_EINVAL, bad
    s = _spec(B)
    s.reserved[1] = 1
    assert B.latent_spec_check(s) == B.MOE_EINVAL


def _cache(B, **kw):
    d = dict(pages=P[0], table=P[1], table_stride=10, n_pages=40, n_seqs=4, max_pages=10, reserved=0)
    d.update(kw)
    return B.MoeLatentCache(*(d[n] for n, _ in B.MoeLatentCache._fields_))


BAD_CACHES = (dict(pages=None), dict(table=None), dict(table_stride=9), dict(n_pages=0), dict(n_seqs=0),
              dict(max_pages=0, table_stride=0), dict(reserved=1), dict(max_pages=1 << 30, table_stride=1 << 30))


def test_append_refusals(B):
    def call(spec=None, cache=None, kv=P[2], gamma=P[3], rope=P[4], max_pos=100, seq=P[5], pos=P[6], T=3, q=P[7], qo=P[8],
             st=P[9]):
        spec, cache = spec or _spec(B), _cache(B) if cache is None else cache
        return B.lib().moe_latent_append(ctypes.byref(spec), ctypes.byref(cache) if cache else None, kv, gamma, rope,
                                         max_pos, seq, pos, T, q, qo, st, None)
    assert call(T=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, heads=0)), dict(cache=False), dict(T=-1), dict(max_pos=0), dict(q=None), dict(qo=None),
                dict(kv=None), dict(gamma=None), dict(rope=None), dict(seq=None), dict(pos=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(cache=_cache(B, pages=P[0] + 8)), dict(kv=P[2] + 8), dict(q=P[7] + 8), dict(rope=P[4] + 4), dict(seq=P[5] + 2),
                dict(st=P[9] + 1)):
        assert call(**bad) == B.MOE_EALIGN, bad


def test_decode_refusals(B):
    def call(spec=None, cache=None, w=P[2], q=P[3], n=2, ln=P[4], most=100, pre=None, plen=0, out=P[5], st=P[6], ws=P[7],
             wb=1 << 40):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent_decode(ctypes.byref(spec), ctypes.byref(cache), w, q, n, ln, most, pre, plen, out, st, ws,
                                         wb, None)
    assert call(n=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, d_v=80)), dict(n=-1), dict(n=5), dict(most=-1), dict(plen=-1), dict(plen=5), dict(w=None), dict(q=None),
                dict(ln=None), dict(out=None), dict(ws=None), dict(most=1 << 27)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(w=P[2] + 2), dict(q=P[3] + 8), dict(ln=P[4] + 2), dict(pre=P[8] + 2, plen=3), dict(out=P[5] + 8), dict(ws=P[7] + 8)):
        assert call(**bad) == B.MOE_EALIGN, bad
    need = B.latent_decode_workspace_bytes(_spec(B), 2, 100)
    assert need > 0 and call(wb=need - 1) == B.MOE_ENOMEM
    assert B.latent_decode_workspace_bytes(_spec(B), 2, 100, 500) > 0
    assert B.latent_decode_workspace_bytes(_spec(B, heads=0), 2, 100) == 0
    assert B.latent_decode_workspace_bytes(_spec(B), -1, 100) == 0


def test_prefill_refusals(B):
    def call(spec=None, cache=None, w=P[2], q=P[3], T=20, qs=P[4], ks=P[5], n=2, kv=50, mq=15, out=P[6], st=P[7], ws=P[8],
             wb=1 << 40):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent_prefill(ctypes.byref(spec), ctypes.byref(cache), w, q, T, qs, ks, n, kv, mq, out, st, ws,
                                          wb, None)
    assert call(T=0, mq=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, d_nope=80)), dict(T=-1), dict(n=-1), dict(n=0), dict(n=5), dict(kv=-1), dict(mq=-1), dict(mq=21),
                dict(mq=0), dict(w=None), dict(q=None), dict(qs=None), dict(ks=None), dict(out=None), dict(ws=None), dict(kv=1 << 25)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(w=P[2] + 2), dict(q=P[3] + 8), dict(qs=P[4] + 2), dict(ks=P[5] + 2), dict(out=P[6] + 8), dict(ws=P[8] + 8)):
        assert call(**bad) == B.MOE_EALIGN, bad
    need = B.latent_prefill_workspace_bytes(_spec(B), 2, 50)
    assert need > 0 and call(wb=need - 1) == B.MOE_ENOMEM


def test_page_call_refusals(B):
    lib = B.lib()

    def copy(pages=P[0], layers=2, lb=1 << 16, pb=1024, n_pages=64, pairs=P[1], n=3, st=P[2]):
        return lib.moe_page_copy(pages, layers, lb, pb, n_pages, pairs, n, st, None)

    assert copy(n=0) == B.MOE_OK
    for bad in (dict(pages=None), dict(layers=0), dict(lb=(1 << 16) - 16), dict(lb=65544), dict(pb=8), dict(pb=1000), dict(n_pages=0),
                dict(pairs=None), dict(n=-1), dict(n=1 << 30)):
        assert copy(**bad) == B.MOE_EINVAL, bad
    assert copy(pages=P[0] + 8) == B.MOE_EALIGN and copy(pairs=P[1] + 4) == B.MOE_EALIGN and copy(st=P[2] + 2) == B.MOE_EALIGN
    assert lib.moe_page_remap(P[0], 0, P[1], 4, P[2], None, None) == B.MOE_OK
    for bad in ((None, 3, P[1], 4, P[2]), (P[0], -1, P[1], 4, P[2]), (P[0], 3, None, 4, P[2]), (P[0], 3, P[1], 0, P[2]),
                (P[0], 3, P[1], 4, None)):
        assert lib.moe_page_remap(*bad, None, None) == B.MOE_EINVAL, bad
    assert lib.moe_page_remap(P[0] + 2, 3, P[1], 4, P[2], None, None) == B.MOE_EALIGN


def test_pool_refusals(B):
    lib, h = B.lib(), ctypes.c_void_p()
    for n, p in ((0, 16), (-1, 16), (1 << 25, 16), (4, 0), (4, 5000)):
        assert lib.moe_page_pool_create(n, p, ctypes.byref(h)) == B.MOE_EINVAL
    assert lib.moe_page_pool_create(4, 16, None) == B.MOE_EINVAL
    for call in (lib.moe_page_pool_destroy, lib.moe_page_pool_available):
        assert call(None) == B.MOE_EINVAL
    pool = B.PagePool(4, 16)
    a = pool.alloc(3)
    assert a == [0, 1, 2] and pool.available() == 1

    def fails(code, fn, *args):
        with pytest.raises(B.MoeError) as e:
            fn(*args)
        assert e.value.code == code
        assert [pool.refs(i) for i in range(4)] == [1, 1, 1, 0] and pool.available() == 1

    fails(B.MOE_ENOMEM, pool.alloc, 2)
    fails(B.MOE_EINVAL, pool.alloc, -1)
    fails(B.MOE_EINVAL, pool.free, [0, 1, 3])
    fails(B.MOE_EINVAL, pool.free, [0, 0])
    fails(B.MOE_EINVAL, pool.free, [0, 4])
    fails(B.MOE_EINVAL, pool.fork, [0, 3], 20)
    fails(B.MOE_EINVAL, pool.fork, [0], -1)
    fails(B.MOE_EINVAL, pool.refs, 4)
    with pytest.raises(ValueError):
        pool.fork([0], 17)
    assert pool.alloc(1) == [3]
    with pytest.raises(B.MoeError) as e:
        pool.fork(a, 40)                         # the last page is partly filled: a page of its own is needed
    assert e.value.code == B.MOE_ENOMEM and [pool.refs(i) for i in range(4)] == [1] * 4
    assert pool.fork(a, 48) == (a, []) and [pool.refs(i) for i in range(4)] == [2, 2, 2, 1]
    pool.free([0, 0, 1, 2])
    assert [pool.refs(i) for i in range(4)] == [0, 1, 1, 1] and pool.available() == 1
    assert pool.fork([], 0) == ([], [])
    pool.close()


@pytest.mark.parametrize("n,page,seed", [(1, 16, 0), (7, 1, 1), (40, 16, 2), (300, 64, 3)])
def test_pool_is_the_oracles(B, n, page, seed):
    g = np.random.default_rng(seed)
    pool, ref = B.PagePool(n, page), A.Pages(n, page)
    seqs = []
    for _ in range(600):
        op = g.integers(5)
        if op <= 1:
            k = int(g.integers(0, max(2, n // 5)))
            want = ref.alloc(k)
            if want is None:
                with pytest.raises(B.MoeError):
                    pool.alloc(k)
            else:
                assert pool.alloc(k) == want
                if k:
                    seqs.append(want)
        elif op == 2 and seqs:
            s = seqs[g.integers(len(seqs))]
            tokens = int(g.integers(0, len(s) * page + 1))
            want = ref.fork(s, tokens)
            if want is None:
                with pytest.raises(B.MoeError):
                    pool.fork(s, tokens)
            else:
                assert pool.fork(s, tokens) == (want[0], want[1])
                if want[0]:
                    seqs.append(want[0])
        elif op == 3 and seqs:
            s = seqs.pop(g.integers(len(seqs)))
            assert ref.free(s)
            pool.free(s)
        elif op == 4 and g.integers(5) == 0:
            moves, remap = ref.compact()
            got, gmap = pool.compact()
            assert [tuple(m) for m in got.tolist()] == moves and gmap.tolist() == remap
            seqs = [[remap[i] for i in s] for s in seqs]
        assert pool.available() == len(ref.free_ids())
        assert [pool.refs(i) for i in range(n)] == ref.refs
    pool.close()


def test_binding_checks(B):
    """What the library cannot see (types, strides, sizes) is refused by the binding, on the CPU."""
    import torch
    pages = torch.zeros(4, 16, 160, dtype=torch.float16)
    with pytest.raises(ValueError):
        B.latent_cache(pages, torch.zeros(2, 3, dtype=torch.int32))       # not on a GPU
    x, y = torch.zeros(2, 128, dtype=torch.float16), torch.zeros(2, 64)
    p = B.MoeProj(P[0], P[1], None, None)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for args in ((x.float(), y), (x, y.double()), (x[:, :64], y), (x, y[:1]), (x, y), (x.t().contiguous().t(), y)):
        with pytest.raises(ValueError):
            B.linear_int4(p, 64, 128, 0, 0.0, *args, ws)
    with pytest.raises(ValueError):
        B.linear_int4(p, 64, 128, 0, 0.0, x, y.half(), ws, add=True)
    with pytest.raises(ValueError):
        B.page_copy(torch.zeros(2, 4, 16), torch.zeros(1, 2, dtype=torch.int32), None)


def test_grids_past_the_launch_limit(B):
    """Calls whose grids would hold 2^32 threads or more are refused before any launch."""
    assert _linear(B, out=1 << 20, ys=1 << 20, T=1 << 18, wb=1 << 40) == B.MOE_EINVAL
    assert B.linear_workspace_bytes(1 << 20, 128, 4, 1 << 18) == 0
    assert B.linear_workspace_bytes(1 << 20, 128, 4, 1 << 17) > 0
    spec, cache = _spec(B, heads=128), _cache(B, n_seqs=1 << 16)
    assert B.lib().moe_latent_prefill(ctypes.byref(spec), ctypes.byref(cache), P[2], P[3], 1 << 16, P[4], P[5], 1 << 16, 1 << 16, 1,
                                      P[6], P[7], P[8], 1 << 60, None) == B.MOE_EINVAL


class _OnGpu:
    """What the binding's checks ask of a tensor, for a device that is not there."""

    is_cuda = True

    def __init__(self, dtype, device=0, contiguous=True):
        self.dtype, self.device, self.contiguous = dtype, device, contiguous

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.device

    def stride(self):
        return (1,)


def test_binding_wants_the_current_device(B, monkeypatch):
    import torch
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    i32 = torch.int32
    B._dense("t", i32, _OnGpu(i32, 1), _OnGpu(i32, 1))
    B._dense("t", i32, _OnGpu(i32, 1), None)
    B._room(_OnGpu(torch.uint8, 1))
    for bad in (_OnGpu(i32, 0), _OnGpu(torch.int64, 1), _OnGpu(i32, 1, False), torch.zeros(2, dtype=i32)):
        for call in (lambda: B._dense("t", i32, bad), lambda: B._dense("t", i32, _OnGpu(i32, 1), None, bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (_OnGpu(i32, 0), _OnGpu(i32, 1, False), torch.zeros(2)):
        with pytest.raises(ValueError):
            B._room(bad)
    with pytest.raises(ValueError):
        B.page_copy(torch.zeros(0, 4, 16), torch.zeros(1, 2, dtype=i32), None)


def test_sequences_of_a_cache(B, monkeypatch):
    """The host's side of a cache: growth, ends and forks of sequences that are not there are refused."""
    import torch
    from paper_2609_18063_amd import latent
    made = {n: getattr(torch, n) for n in ("zeros", "full")}
    for n, f in made.items():
        monkeypatch.setattr(torch, n, lambda *a, _f=f, device=None, **k: _f(*a, **k))
    monkeypatch.setattr(B, "latent_cache", lambda pages, table: None)
    cache = latent.LatentCache(_spec(B), 1, 6, 3, 64)
    a = cache.start()
    assert cache.grow(a, 0) == 0 and cache.grow(a, 32) == 0 and cache.grow(a, 16) == 32
    for call in (lambda: cache.grow(a, -1), lambda: cache.grow(1, 1), lambda: cache.grow(3, 1), lambda: cache.grow(-1, 1),
                 lambda: cache.end(1), lambda: cache.fork(2), lambda: cache.grow(a, 17)):
        with pytest.raises(ValueError):
            call()
    assert cache.ids == [[0, 1, 2], None, None] and cache.tokens == [48, 0, 0] and cache.pool.available() == 3
    b = cache.fork(a)                                     # (48 tokens: whole pages, nothing to copy)
    assert cache.ids[b] == [0, 1, 2] and cache.pool.refs(1) == 2
    cache.grow(b, 1)
    cache.end(a)
    assert cache.table[a].tolist() == [-1] * 4 and cache.table[b].tolist() == [0, 1, 2, 3]
    with pytest.raises(ValueError):
        cache.end(a)
    c = cache.start()
    assert c == a
    cache.grow(c, 32)
    with pytest.raises(B.MoeError):
        cache.grow(c, 32)                                 # two more pages than are free: nothing changes
    assert cache.ids[c] == [4, 5] and cache.tokens[c] == 32 and cache.table[c].tolist() == [4, 5, -1, -1]
    cache.close()
