"""The attention block on padded batches: rows of padding keep their residual."""

import numpy as np
import pytest

from oracle import attention as A
from tests.test_gpu_attention_chain import DR, _blocks, _close, _oracle, _spec

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
