"""The attention oracle against itself: the absorbed and the expanded form give the same output, a query that
sees one token gives that token's value, and pages are counted as a brute-force list of sequences says."""

import numpy as np
import pytest

from oracle import attention as A, quant


@pytest.mark.parametrize("L,n", [(1, 1), (7, 3), (200, 9)])
def test_absorbed_is_expanded(L, n):
    g = np.random.default_rng(L)
    Dc, Dr, Dn, Dv = 24, 8, 16, 12
    rows, q = g.standard_normal((L, Dc + Dr)), g.standard_normal((n, Dn + Dr))
    uk, uv = g.standard_normal((Dn, Dc)), g.standard_normal((Dv, Dc))
    seen = g.integers(1, L + 1, n)
    got, _ = A.attend(q, rows, uk, uv, 0.3, seen)
    k, v = np.concatenate([rows[:, :Dc] @ uk.T, rows[:, Dc:]], -1), rows[:, :Dc] @ uv.T
    for i in range(n):
        s = 0.3 * k[:seen[i]] @ q[i]
        p = np.exp(s - s.max())
        assert np.allclose(got[i], p @ v[:seen[i]] / p.sum(), rtol=1e-12, atol=1e-12)


def test_one_token_and_none():
    g = np.random.default_rng(1)
    rows, uk, uv = g.standard_normal((5, 12)), g.standard_normal((4, 8)), g.standard_normal((6, 8))
    o, b = A.attend(g.standard_normal((2, 8)), rows, uk, uv, 1.0, np.array([1, 0]))
    assert np.allclose(o[0], uv @ rows[0, :8]) and not o[1].any() and not b[1].any() and (b[0] > 0).all()


def test_projection_is_dense():
    g = np.random.default_rng(2)
    codes = g.integers(0, 16, (5, 128)).astype(np.uint8)
    s, z = g.standard_normal((5, 2)).astype(np.float16), g.standard_normal((5, 2)).astype(np.float16)
    a, b, x = g.standard_normal((3, 128)), g.standard_normal((5, 3)), g.standard_normal((4, 128))
    y, mag = A.projection((quant.pack_nibbles(codes), s, z), (a, b), 1.5, x)
    w = np.repeat(s, 64, 1).astype(np.float64) * codes + np.repeat(z, 64, 1)
    assert np.allclose(y, x @ (w + 1.5 * b @ a).T) and (mag >= np.abs(y) - 1e-9).all()


def test_row_norm_and_rotation():
    g = np.random.default_rng(3)
    t = A.rope_table(50, 8)
    kv = g.standard_normal((3, 24))
    row = A.cache_row(kv, np.ones(16), t[7, :, 0], t[7, :, 1])
    assert np.allclose((row[:, :16] ** 2).mean(-1), 1, atol=1e-5)
    assert np.allclose(np.linalg.norm(row[:, 16:], axis=-1), np.linalg.norm(kv[:, 16:], axis=-1), rtol=1e-6)
    z = (kv[:, 16::2] + 1j * kv[:, 17::2]) * np.exp(1j * np.arccos(np.clip(t[7, :, 0], -1, 1)) * np.sign(t[7, :, 1]))
    assert np.allclose(row[:, 16::2] + 1j * row[:, 17::2], z, atol=1e-3)


def test_pages_by_sequences():
    """Random forks, frees and compactions: a page's references are the sequences that hold it."""
    g = np.random.default_rng(4)
    P = A.Pages(40, 16)
    seqs, size = {}, {}
    for step in range(400):
        op = g.integers(4)
        if op == 0:
            n = int(g.integers(1, 80))
            ids = P.alloc(-(-n // 16))
            if ids is not None:
                seqs[step], size[step] = ids, n
        elif op == 1 and seqs:
            k = list(seqs)[g.integers(len(seqs))]
            n = int(g.integers(1, size[k] + 1))
            got = P.fork(seqs[k][:-(-n // 16)], n)
            if got is not None:
                seqs[step], size[step] = got[0], n
        elif op == 2 and seqs:
            k = list(seqs)[g.integers(len(seqs))]
            assert P.free(seqs.pop(k))
        elif op == 3:
            moves, remap = P.compact()
            seqs = {k: [remap[i] for i in v] for k, v in seqs.items()}
            live = sum(r > 0 for r in P.refs)
            assert all(P.refs[i] > 0 for i in range(live))
            assert not {a for a, _ in moves} & {b for _, b in moves}
        count = [0] * 40
        for v in seqs.values():
            for i in v:
                count[i] += 1
        assert count == P.refs
