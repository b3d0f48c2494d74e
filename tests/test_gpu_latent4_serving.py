"""The 4-bit cache's calls together, as programs use them: a serving run of prompts in chunks, single tokens, forks,
evictions and a compaction, and a decode chain whose layers attend over such a cache. Every step is checked against the
float64 oracle on the device's own inputs of that step and on the rows that the cache says it holds.

Tolerance, in the norm of an output: as of the fp16 cache's run, with the cached values' rounding to fp16 as an operand
in the place of the cache row's (which here is part of what the cache holds): 16 A.HALF."""

import numpy as np
import pytest

import synth
from oracle import attention as A, routing as o_routing
from tests.gpu_harness import build_chain
from tests.test_gpu_attention_chain import DC, DN, DR, DV, H, _blocks, _close, _project, _spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _step(block, x, pos, rows, rope):
    """(outputs, new rows, weights of all tokens) of the last len(x) tokens of ``rows``, at positions ``pos``."""
    cs = rope[pos].astype(np.float64)
    new = A.cache_row(_project(block["kv"], x), block["gamma"], cs[..., 0], cs[..., 1])
    q = _project(block["q"], x).reshape(len(x), H, DN + DR)
    q = np.concatenate([q[..., :DN], A.rotate(q[..., DN:], cs[:, None, :, 0], cs[:, None, :, 1])], -1)
    seen = np.arange(len(rows) - len(x), len(rows)) + 1
    scale = 1 / np.sqrt(DN + DR)
    o = np.stack([A.attend(q[:, h], rows, block["w"][h, :DN], block["w"][h, DN:], scale, seen)[0] for h in range(H)], 1)
    w, _ = A.token_weights(q, rows, block["w"][:, :DN], scale, seen)
    return _project(block["o"], o.reshape(len(x), H * DV)), new, w


def _is_quantized(got, want):
    """A cached row's groups are within half a step of the values, and a tenth for all the other roundings (s, z, fp32
    projections and the value's to fp16, which are under a hundredth of a step each)."""
    for a in range(0, DC + DR, 64):
        x = want[:, a:a + 64]
        step = (x.max(-1) - x.min(-1))[:, None] / 15
        assert (np.abs(got[:, a:a + 64] - x) <= 0.6 * step).all()


def test_serving_run(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(5)
    from paper_2609_18063_amd import latent
    d, L, page, most = 256, 2, 16, 160
    spec = _spec(page)
    dev, host = _blocks(torch, d, L, 31)
    cache = latent.LatentCache(spec, L, 48, 4, most, bits=4, weights=True)
    attn = latent.LatentAttention(d, spec, dev, cache, latent.rope_table(400, DR), max_rows=64)
    rope = A.rope_table(400, DR)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    sums = {}                                             # (layer, sequence): its sums, float64

    def check(layer, b, x, got, pos, what):
        rows = cache.rows(layer, b).cpu().numpy().astype(np.float64)
        want, new, w = _step(host[layer], x, pos, rows, rope)
        _close(got, want, (what, layer, b))
        _is_quantized(rows[len(rows) - len(x):], new)
        w[:len(sums.get((layer, b), []))] += sums.get((layer, b), [])
        sums[layer, b] = w
        now = cache.sums[layer, b].cpu().numpy()
        _close(now[:len(w)], w, (what, "sums", layer, b))
        assert not now[len(w):].any()

    def chunk(counts):
        """A prefill of counts[b] more tokens of sequences 0 .. len(counts) - 1."""
        first = [cache.grow(b, n) for b, n in enumerate(counts)]
        T = sum(counts)
        qs, ks = np.concatenate([[0], np.cumsum(counts)]), np.concatenate([[0], np.cumsum(cache.tokens[:len(counts)])])
        seq = np.repeat(np.arange(len(counts)), counts)
        slot = np.concatenate([np.arange(a, a + n) for a, n in zip(first, counts)])
        pos = slot + np.repeat([cache.evicted[b] for b in range(len(counts))], counts)
        for layer in range(L):
            x, r0 = g.standard_normal((T, d)).astype(np.float16), g.standard_normal((T, d)).astype(np.float32)
            r = torch.from_numpy(r0).cuda()
            attn.prefill(layer, torch.from_numpy(x).cuda(), r, i32(seq), i32(pos), i32(qs), i32(ks), int(ks[-1]), max(counts),
                         slot=i32(slot))
            got = r.cpu().numpy().astype(np.float64) - r0
            for b, n in enumerate(counts):
                if n:
                    check(layer, b, x[qs[b]:qs[b + 1]], got[qs[b]:qs[b + 1]], pos[qs[b]:qs[b + 1]], "chunk")

    def step(live):
        """One token of each live sequence, in a batch of all table rows."""
        n = len(cache.ids)
        slot = [cache.grow(b, 1) if b in live else 0 for b in range(n)]
        pos = [p + cache.evicted[b] for b, p in enumerate(slot)]
        seq, kv = [b if b in live else -1 for b in range(n)], [p + 1 if b in live else 0 for b, p in enumerate(slot)]
        for layer in range(L):
            x, r0 = g.standard_normal((n, d)).astype(np.float16), g.standard_normal((n, d)).astype(np.float32)
            r = torch.from_numpy(r0).cuda()
            attn.decode(layer, torch.from_numpy(x).cuda(), r, i32(seq), i32(pos), i32(kv), slot=i32(slot))
            got = r.cpu().numpy().astype(np.float64) - r0
            for b in range(n):
                if b not in live:
                    assert not got[b].any(), b             # a padding row's residual stays as it was
                else:
                    check(layer, b, x[b:b + 1], got[b:b + 1], np.array([pos[b]]), "step")

    def evict(budget, sinks, recent):
        was = {k: cache.rows(*k).cpu().numpy() for k in sums}
        own = {k: cache.sums[k].cpu().numpy() for k in sums}
        tokens = list(cache.tokens)
        gone = cache.evict(budget, sinks, recent)
        for (layer, b), rows in was.items():
            ids = A.evict(own[layer, b], tokens[b], budget, sinks, recent)
            assert gone[b] == tokens[b] - len(ids) and cache.tokens[b] == len(ids)
            assert np.array_equal(cache.rows(layer, b).cpu().numpy(), rows[ids])
            assert np.array_equal(cache.sums[layer, b].cpu().numpy()[:len(ids)], own[layer, b][ids])
            sums[layer, b] = sums[layer, b][ids]
        return gone

    assert [cache.start() for _ in range(2)] == [0, 1]
    chunk([45, 16])
    chunk([19, 3])
    new = cache.fork(0)
    for layer in range(L):
        sums[layer, new] = sums[layer, 0].copy()
    step({0, 1, new})
    assert evict(40, 2, 8) == [25, 0, 25, 0]               # the fork and its origin share their pages
    step({0, 1, new})
    chunk([23, 30])
    step({0, 1, new})
    assert evict(33, 0, 1) == [65 - 33, 52 - 33, 42 - 33, 0]
    assert cache.compact() > 0
    for _ in range(18):                                    # on past a page's end
        step({0, 1, new})
    cache.end(1)
    for layer in range(L):
        del sums[layer, 1]
    assert cache.start() == 1
    chunk([0, 40])
    step({0, 1, new})
    assert evict(200, 5, 5) == [0, 0, 0, 0]
    assert int(cache.status) == 0
    for bad in ((0, 0, 0), (5, 3, 3), (5, -1, 2)):
        with pytest.raises(ValueError):
            cache.evict(*bad)
    third = cache.fork(new)
    for s in (0, 1, new, third):
        cache.end(s)
    assert cache.pool.available() == 48
    cache.close()


def test_evict_without_free_pages(torch_cuda):
    """Nothing changes where the pool cannot give the new pages; a cache without sums refuses."""
    from paper_2609_18063_amd import binding as B, latent
    cache = latent.LatentCache(_spec(16), 1, 4, 1, 64, bits=4, weights=True)
    cache.grow(cache.start(), 64)
    with pytest.raises(B.MoeError) as e:
        cache.evict(10)
    assert e.value.code == B.MOE_ENOMEM and cache.tokens == [64] and cache.ids == [[0, 1, 2, 3]] and cache.evicted == [0]
    cache.close()
    for kw in (dict(bits=8), dict(weights=True)):
        with pytest.raises(ValueError):
            latent.LatentCache(_spec(16), 1, 4, 1, 64, **kw)
    plain = latent.LatentCache(_spec(16), 1, 4, 1, 64, bits=4)
    with pytest.raises(ValueError):
        plain.evict(10)
    plain.close()


def test_decode_chain_on_four_bits(torch_cuda):
    torch = torch_cuda
    from paper_2609_18063_amd import chain as C, latent
    wl, L, T = synth.WORKLOADS["tiny"], 3, 20
    plain, _ = build_chain(wl, L, torch)
    dev, host = _blocks(torch, wl.d, L, 77)
    attn = latent.ChainAttention(wl.d, _spec(16), dev, T, bits=4)
    chain = C.DeviceChain(plain.spec, plain.table, plain.layers, attention=attn)
    xi = torch.from_numpy(synth.token_draws(wl, 0, T)).cuda()
    rec = {k: v.cpu().numpy() for k, v in chain.run_recorded(xi).items()}
    assert int(chain.status) == 0 and int(attn.cache.status) == 0
    rope = A.rope_table(T, DR)
    for n in range(L):
        rows = attn.cache.rows(n, 0).cpu().numpy().astype(np.float64)
        for t in range(T):
            x = o_routing.rms_norm_f16(rec["r_in"][t, n])[None]
            want, new, _ = _step(host[n], x, np.array([t]), rows[:t + 1], rope)
            _close(rec["r"][t, n].astype(np.float64) - rec["r_in"][t, n], want[0], (t, n))
            _is_quantized(rows[t:t + 1], new)
    # the captured token graphs, twice over the tokens, with the eager chain's own work between them
    chain.capture()
    for again in range(2):
        chain.reset()
        for t in range(T):
            chain.xi.copy_(xi[t:t + 1])
            chain.replay_token(t)
            assert np.array_equal(chain.r[0].cpu().numpy(), rec["r_post"][t, L - 1]), (again, t)
    plain.table.close()
