"""The attention block on padded batches and shared prefixes: rows of padding keep their residual, and a sequence's own
tokens stand behind whole pages that others share."""

import numpy as np
import pytest

from oracle import attention as A
from tests.test_gpu_attention_chain import DC, DN, DR, DV, H, _blocks, _close, _oracle, _spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def test_padded_prompts(torch_cuda):
    """Rows behind the last sequence (seq -1), after a call whose outputs lay there, and with NaN in their inputs."""
    torch, g = torch_cuda, np.random.default_rng(61)
    from paper_2609_18063_amd import latent
    d, page, most = 256, 16, 96
    dev, host = _blocks(torch, d, 1, 41)
    cache = latent.LatentCache(_spec(page), 1, 20, 2, most)
    attn = latent.LatentAttention(d, _spec(page), dev, cache, latent.rope_table(most, DR), max_rows=64)
    attn.ob.fill_(float("nan"))                            # (no initial contents are promised)
    rope = A.rope_table(most, DR)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    a, b = cache.start(), cache.start()
    rows = {a: [], b: []}
    for counts, T in (((20, 7), 40), ((30, 21), 51), ((5, 2), 64)):
        first = [cache.grow(s, n) for s, n in zip((a, b), counts)]
        live = sum(counts)
        qs, ks = np.concatenate([[0], np.cumsum(counts)]), np.concatenate([[0], np.cumsum(cache.tokens)])
        seq = np.concatenate([np.repeat([a, b], counts), np.full(T - live, -1)])
        pos = np.concatenate([np.arange(at, at + n) for at, n in zip(first, counts)] + [np.zeros(T - live, int)])
        x, r0 = g.standard_normal((T, d)).astype(np.float16), g.standard_normal((T, d)).astype(np.float32)
        x[live:] = np.nan
        r = torch.from_numpy(r0).cuda()
        attn.prefill(0, torch.from_numpy(x).cuda(), r, i32(seq), i32(pos), i32(qs), i32(ks), int(ks[-1]), max(counts))
        got = r.cpu().numpy()
        assert np.array_equal(got[live:], r0[live:]), counts
        for s, part in ((a, slice(0, counts[0])), (b, slice(counts[0], live))):
            want, rows[s] = _oracle(host[0], x[part], pos[part], rows[s], rope)
            _close(got[part].astype(np.float64) - r0[part], want, (counts, s))
    assert int(cache.status) == 0
    cache.close()


def test_own_tokens_behind_a_shared_prefix(torch_cuda):
    """The prefix's pages stand first in every table row, so that positions are the tokens' own; the attention takes them
    as the prefix, and the table from the column behind them."""
    torch, g = torch_cuda, np.random.default_rng(62)
    from paper_2609_18063_amd import binding as B, latent
    page, whole, own, n = 16, 5, 40, 3
    prefix, most = whole * page, whole * page + own
    spec = _spec(page)
    cache = latent.LatentCache(spec, 1, 30, n + 1, most)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    base = cache.start()
    cache.grow(base, prefix)
    ids = cache.ids[base]
    seqs = [cache.fork(base) for _ in range(n)]
    assert all(cache.ids[s][:whole] == ids for s in seqs)  # (whole pages: shared, none copied)
    rope, gamma = latent.rope_table(most, DR), (1 + 0.1 * g.standard_normal(DC)).astype(np.float16)
    turn = A.rope_table(most, DR).astype(np.float64)
    w = (g.standard_normal((H, DN + DV, DC)) / np.sqrt(DC)).astype(np.float16)
    wt, gt = torch.from_numpy(w).cuda(), torch.from_numpy(gamma).cuda()

    def append(seq, pos, q=None):
        kv = g.standard_normal((len(seq), DC + DR)).astype(np.float32)
        out = None if q is None else torch.empty_like(q)
        B.latent_append(spec, cache.layers[0], torch.from_numpy(kv).cuda(), gt, rope, i32(seq), i32(pos), cache.status, q=q, q_out=out)
        return A.cache_row(kv, gamma, turn[pos, :, 0], turn[pos, :, 1]), out

    first, _ = append([base] * prefix, np.arange(prefix))
    rows = {s: first for s in seqs}
    views = B.latent_cache(cache.pages[0], cache.table[1:, whole:])
    ws = torch.empty(B.latent_decode_workspace_bytes(spec, n, own, prefix), dtype=torch.uint8, device="cuda")
    out = torch.empty(n, H, DV, dtype=torch.float16, device="cuda")
    assert seqs == [1, 2, 3]
    for step in range(35):
        pos = np.array([cache.grow(s, 1) for s in seqs])
        q = torch.from_numpy((1.5 * g.standard_normal((n, H, DN + DR))).astype(np.float16)).cuda()
        new, q = append(seqs, pos, q)
        for k, s in enumerate(seqs):
            rows[s] = np.concatenate([rows[s], new[k:k + 1]])
        B.latent_decode(spec, views, wt, q, i32([step + 1] * n), own, out, cache.status, ws, prefix=i32(ids), prefix_len=prefix)
        if step % 5 and step < 30:
            continue
        got, qn = out.cpu().numpy().astype(np.float64), q.cpu().numpy()
        for k, s in enumerate(seqs):
            want = np.stack([A.attend(qn[k:k + 1, h], rows[s], w[h, :DN], w[h, DN:], 1 / np.sqrt(DN + DR))[0][0] for h in range(H)])
            _close(got[k], want, (step, s))
    assert int(cache.status) == 0
    cache.close()
