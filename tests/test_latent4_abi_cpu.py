"""Argument checks of the 4-bit cache's and the eviction's calls, without a GPU (the device addresses below are never
dereferenced: a refused call enqueues nothing), and the oracle's own rows."""

import ctypes

import numpy as np
import pytest

from oracle import attention as A
from tests.test_attention_abi_cpu import BAD_CACHES, P, _cache, _spec


@pytest.fixture(scope="module")
def B():
    from paper_2609_18063_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("Dc,Dr,page,want", [(512, 64, 64, 64 * 324), (512, 64, 16, 16 * 324), (128, 32, 16, 16 * 92), (256, 32, 1024, 1024 * 164)])
def test_page_bytes(B, Dc, Dr, page, want):
    assert B.latent4_page_bytes(_spec(B, d_latent=Dc, d_rope=Dr, page_tokens=page)) == want
    assert A.Pages4(1, page, Dc, Dr).raw.shape[1] == want
    assert B.latent4_page_bytes(_spec(B, heads=0)) == 0


def test_append_and_read_refusals(B):
    def call(spec=None, cache=None, kv=P[2], gamma=P[3], rope=P[4], max_pos=100, seq=P[5], slot=P[10], pos=P[6], T=3, q=P[7],
             qo=P[8], st=P[9]):
        spec, cache = spec or _spec(B), _cache(B) if cache is None else cache
        return B.lib().moe_latent4_append(ctypes.byref(spec), ctypes.byref(cache) if cache else None, kv, gamma, rope,
                                          max_pos, seq, slot, pos, T, q, qo, st, None)
    assert call(T=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, heads=0)), dict(cache=False), dict(T=-1), dict(T=(1 << 22) + 1), dict(max_pos=0), dict(q=None), dict(qo=None),
                dict(kv=None), dict(gamma=None), dict(rope=None), dict(seq=None), dict(slot=None), dict(pos=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(cache=_cache(B, pages=P[0] + 8)), dict(kv=P[2] + 8), dict(q=P[7] + 8), dict(rope=P[4] + 4), dict(seq=P[5] + 2),
                dict(slot=P[10] + 2), dict(pos=P[6] + 1), dict(st=P[9] + 1)):
        assert call(**bad) == B.MOE_EALIGN, bad

    def read(spec=None, cache=None, seq=P[2], slot=P[3], T=3, rows=P[4], st=P[5]):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent4_read(ctypes.byref(spec), ctypes.byref(cache), seq, slot, T, rows, st, None)
    assert read(T=0) == B.MOE_OK
    for bad in (dict(spec=_spec(B, d_rope=16)), dict(T=-1), dict(T=1 << 25), dict(seq=None), dict(slot=None), dict(rows=None)):
        assert read(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(seq=P[2] + 2), dict(slot=P[3] + 2), dict(rows=P[4] + 8), dict(st=P[5] + 2)):
        assert read(**bad) == B.MOE_EALIGN, bad


def test_decode_refusals(B):
    def call(spec=None, cache=None, w=P[2], q=P[3], n=2, ln=P[4], most=100, out=P[5], sums=P[8], stride=100, st=P[6], ws=P[7],
             wb=1 << 40):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent4_decode(ctypes.byref(spec), ctypes.byref(cache), w, q, n, ln, most, out, sums, stride, st, ws,
                                          wb, None)
    assert call(n=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, d_v=80)), dict(n=-1), dict(n=5), dict(most=-1), dict(w=None), dict(q=None), dict(ln=None),
                dict(out=None), dict(ws=None), dict(most=1 << 27, stride=1 << 28), dict(stride=99), dict(stride=-1)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(w=P[2] + 2), dict(q=P[3] + 8), dict(ln=P[4] + 2), dict(out=P[5] + 8), dict(ws=P[7] + 8), dict(sums=P[8] + 2),
                dict(st=P[6] + 2)):
        assert call(**bad) == B.MOE_EALIGN, bad
    for sums in (False, True):
        need = B.latent4_decode_workspace_bytes(_spec(B), 2, 100, sums)
        assert need > 0 and call(wb=need - 1, sums=P[8] if sums else None) == B.MOE_ENOMEM
    assert B.latent4_decode_workspace_bytes(_spec(B, heads=0), 2, 100) == 0
    assert B.latent4_decode_workspace_bytes(_spec(B), -1, 100) == 0


def test_prefill_refusals(B):
    def call(spec=None, cache=None, w=P[2], q=P[3], T=20, qs=P[4], ks=P[5], n=2, kv=50, mq=15, out=P[6], sums=P[9], stride=30, room=30,
             st=P[7], ws=P[8], wb=1 << 40):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent4_prefill(ctypes.byref(spec), ctypes.byref(cache), w, q, T, qs, ks, n, kv, mq, out, sums, stride,
                                           room, st, ws, wb, None)
    assert call(T=0, mq=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert call(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, d_nope=80)), dict(T=-1), dict(n=-1), dict(n=0), dict(n=5), dict(kv=-1), dict(mq=-1), dict(mq=21),
                dict(mq=0), dict(w=None), dict(q=None), dict(qs=None), dict(ks=None), dict(out=None), dict(ws=None),
                dict(kv=1 << 25), dict(stride=29), dict(room=0), dict(stride=-1)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(w=P[2] + 2), dict(q=P[3] + 8), dict(qs=P[4] + 2), dict(ks=P[5] + 2), dict(out=P[6] + 8), dict(ws=P[8] + 8),
                dict(sums=P[9] + 2)):
        assert call(**bad) == B.MOE_EALIGN, bad
    for sums in (False, True):
        need = B.latent4_prefill_workspace_bytes(_spec(B), 20, 2, 50, sums)
        assert need > 0 and call(wb=need - 1, sums=P[9] if sums else None) == B.MOE_ENOMEM
    rows = -(-50 * (_spec(B).d_latent + _spec(B).d_rope) * 2 // 256) * 256  # the context's rows as fp16
    assert B.latent4_prefill_workspace_bytes(_spec(B), 20, 2, 50) == B.latent_prefill_workspace_bytes(_spec(B), 2, 50) + rows


def test_evict_refusals(B):
    def select(sums=P[0], out=P[1], layers=2, n=3, width=50, ln=P[2], budget=10, sinks=2, recent=8, keep=P[3], st=P[4]):
        return B.lib().moe_evict_select(sums, out, layers, n, width, ln, budget, sinks, recent, keep, st, None)
    assert select(n=0) == B.MOE_OK
    for bad in (dict(sums=None), dict(out=None), dict(layers=0), dict(n=-1), dict(width=0), dict(width=1 << 27), dict(ln=None),
                dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(recent=9), dict(keep=None), dict(layers=1 << 20, n=1 << 10),
                dict(sinks=(1 << 31) - 1, recent=(1 << 31) - 1)):
        assert select(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(sums=P[0] + 2), dict(out=P[1] + 2), dict(ln=P[2] + 1), dict(keep=P[3] + 2), dict(st=P[4] + 2)):
        assert select(**bad) == B.MOE_EALIGN, bad

    def move(spec=None, cache=None, layers=2, lb=40 * 16 * 92, keep=P[2], n=2, budget=33, to=P[3], ts=3, st=P[4]):
        spec, cache = spec or _spec(B), cache or _cache(B)
        return B.lib().moe_latent4_move(ctypes.byref(spec), ctypes.byref(cache), layers, lb, keep, n, budget, to, ts, st, None)
    assert move(n=0) == B.MOE_OK
    for c in BAD_CACHES:
        assert move(cache=_cache(B, **c)) == B.MOE_EINVAL, c
    for bad in (dict(spec=_spec(B, heads=0)), dict(layers=0), dict(layers=65536), dict(lb=40 * 16 * 92 - 16), dict(lb=40 * 16 * 92 + 8),
                dict(keep=None), dict(n=-1), dict(n=5), dict(budget=0), dict(to=None), dict(ts=2)):
        assert move(**bad) == B.MOE_EINVAL, bad
    assert move(keep=P[2] + 2) == B.MOE_EALIGN and move(to=P[3] + 2) == B.MOE_EALIGN and move(st=P[4] + 1) == B.MOE_EALIGN


def test_oracle_rows():
    """A group's values come back within half a step and the roundings of s and z; its ends within them alone."""
    g = np.random.default_rng(0)
    v = g.standard_normal((50, 128 + 32)) * np.exp(g.standard_normal((50, 1)))
    v[3] = 0.25
    codes, s, z = A.quantize_row(v, 128)
    back = A.row_values(codes, s, z, 128)
    grp = np.minimum(np.arange(160) // 64, 2)
    step = s.astype(np.float64)[:, grp]
    assert (np.abs(back - v) <= step * (0.5 + 8 * A.HALF) + A.HALF * np.abs(z.astype(np.float64))[:, grp] + 16 * A.TINY).all()
    assert np.array_equal(back[3], v[3]) and (codes[3] == 8).all()
    mem = A.Pages4(3, 16, 128, 32)
    page, at = np.array([2, 0, 2]), np.array([5, 15, 0])
    mem.put(page, at, codes[:3], s[:3], z[:3])
    for a, b in zip(mem.get(page, at), (codes, s, z)):
        assert np.array_equal(a, b[:3])


def test_oracle_evicts():
    assert A.evict(np.array([5, 1, 1, 9, 1, 2.0]), 6, 4, 1, 1) == [0, 1, 3, 5]
    assert A.evict(np.array([0, np.nan, 1.0]), 3, 1, 0, 0) == [2] and A.evict(np.array([1.0, 2]), 2, 3, 1, 1) == [0, 1]


@pytest.mark.parametrize("H", [1, 17, 33, 64, 65, 128])
@pytest.mark.parametrize("dims", [(128, 32), (256, 64), (512, 64)])
def test_a_larger_calls_workspace_does_for_a_smaller_one(B, H, dims):
    """A serving loop keeps one for its largest batch and longest context."""
    spec = B.make_latent_spec(H, *dims, 64, 64, 64, 0.1)
    for sums in (False, True):
        v = [(b, n, B.latent4_decode_workspace_bytes(spec, b, n, sums))
             for b in (1, 2, 9, 64, 300, 5000) for n in (0, 1, 65, 769, 5000, 12000, 16384, 50000, 400000, 1 << 20)]
        assert all(y <= x for b, n, x in v for b2, n2, y in v if b2 <= b and n2 <= n)
