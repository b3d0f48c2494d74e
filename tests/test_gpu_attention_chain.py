"""The attention block's calls together, as programs use them: a decode chain whose layers attend over a paged
cache (eager and replayed from graphs), and a serving run of prompts in chunks, forks, a padded batch and a
compaction. Every step is checked against the float64 oracle on the device's own inputs of that step.

Tolerance, in the norm of a layer's output: seven values on the way are rounded to fp16 (the query, its rotation,
the cache row, the query in the latent space or the keys, the weights, the latents or the values, the output),
each by at most A.HALF; the first four move scores of up to about 4 in size by as much, 4 (first four) x 3 for the
softmax's two-sided effect at rms scores near 1.5 would be 12, and 3 more: 16 A.HALF bounds it with fp32 sums."""

import numpy as np
import pytest

import synth
from oracle import attention as A, routing as o_routing
from tests.gpu_harness import build_chain

pytestmark = pytest.mark.gpu
TOL = 16 * A.HALF


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


H, DC, DR, DN, DV, RANK, SCALE = 4, 128, 32, 64, 64, 8, 2.0


def _spec(page):
    from paper_2609_18063_amd import binding as B
    return B.make_latent_spec(H, DC, DR, DN, DV, page, 1 / np.sqrt(DN + DR))


def _blocks(torch, d, n_layers, seed):
    from paper_2609_18063_amd import binding as B, latent
    dev, host = [], []
    for n in range(n_layers):
        g, projs, keep, np_projs = np.random.default_rng(seed + n), [], [], []
        for k, (o, i) in enumerate(((H * (DN + DR), d), (DC + DR, d), (d, H * DV))):
            qsz = synth.int4_projection((seed, n, k, 0), (seed, n, k, 1), o, i, w_std=1 / np.sqrt(i))
            lora = synth.lora_pair((seed, n, k, 2), (seed, n, k, 3), o, i, RANK, 1 / RANK, 0.01)
            p, kp = B.upload_projection(qsz, lora, "cuda")
            projs.append(p)
            keep += kp
            np_projs.append((qsz, lora))
        w = (g.standard_normal((H, DN + DV, DC)) / np.sqrt(DC)).astype(np.float16)
        gamma = (1 + 0.1 * g.standard_normal(DC)).astype(np.float16)
        dev.append(latent.LatentBlock(*projs, torch.from_numpy(w).cuda(), torch.from_numpy(gamma).cuda(), RANK, SCALE, keep))
        host.append({"q": np_projs[0], "kv": np_projs[1], "o": np_projs[2], "w": w, "gamma": gamma})
    return dev, host


def _project(p, x):
    return A.projection(p[0], p[1], SCALE, x)[0]


def _oracle(block, x, pos, rows_before, rope):
    """Outputs of the tokens ``x`` at ``pos`` that follow ``rows_before`` in their sequence, and their rows."""
    cs = rope[pos].astype(np.float64)
    rows = A.cache_row(_project(block["kv"], x), block["gamma"], cs[..., 0], cs[..., 1])
    q = _project(block["q"], x).reshape(len(x), H, DN + DR)
    q = np.concatenate([q[..., :DN], A.rotate(q[..., DN:], cs[:, None, :, 0], cs[:, None, :, 1])], -1)
    every = np.concatenate([rows_before, rows]) if len(rows_before) else rows
    seen = len(rows_before) + np.arange(len(x)) + 1
    o = np.stack([A.attend(q[:, h], every, block["w"][h, :DN], block["w"][h, DN:], 1 / np.sqrt(DN + DR), seen)[0]
                  for h in range(H)], 1)
    return _project(block["o"], o.reshape(len(x), H * DV)), every


def _close(got, want, what):
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert off <= TOL, (what, off)


def test_decode_chain_with_attention(torch_cuda):
    torch = torch_cuda
    from paper_2609_18063_amd import chain as C, latent
    wl, L, T = synth.WORKLOADS["tiny"], 3, 20
    plain, _ = build_chain(wl, L, torch)
    dev, host = _blocks(torch, wl.d, L, 77)
    attn = latent.ChainAttention(wl.d, _spec(16), dev, T)
    chain = C.DeviceChain(plain.spec, plain.table, plain.layers, attention=attn)
    xi = torch.from_numpy(synth.token_draws(wl, 0, T)).cuda()
    rec = {k: v.cpu().numpy() for k, v in chain.run_recorded(xi).items()}
    assert int(chain.status) == 0 and int(attn.cache.status) == 0
    rope = A.rope_table(T, DR)
    for n in range(L):
        rows = np.zeros((0, DC + DR))
        for t in range(T):
            x = o_routing.rms_norm_f16(rec["r_in"][t, n])[None]
            want, rows = _oracle(host[n], x, np.array([t]), rows, rope)
            _close(rec["r"][t, n].astype(np.float64) - rec["r_in"][t, n], want[0], (t, n))
            assert np.array_equal(rec["x"][t, n], o_routing.rms_norm_f16(rec["r"][t, n])), (t, n)
    # the captured token graphs, twice over the tokens, with the eager chain's own work between them
    chain.capture()
    for again in range(2):
        chain.reset()
        for t in range(T):
            chain.xi.copy_(xi[t:t + 1])
            chain.replay_token(t)
            assert np.array_equal(chain.r[0].cpu().numpy(), rec["r_post"][t, L - 1]), (again, t)
    with pytest.raises(ValueError):
        attn.at(T)
    plain.table.close()


def test_serving_run(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(5)
    from paper_2609_18063_amd import latent
    d, L, page, most = 256, 2, 16, 160
    spec = _spec(page)
    dev, host = _blocks(torch, d, L, 31)
    cache = latent.LatentCache(spec, L, 40, 4, most)
    attn = latent.LatentAttention(d, spec, dev, cache, latent.rope_table(most, DR), max_rows=64)
    rope = A.rope_table(most, DR)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    rows = {}                                             # (layer, sequence): its rows, float64

    def draw(n):
        return g.standard_normal((n, d)).astype(np.float16)

    def chunk(counts):
        """A prefill of counts[b] more tokens of sequences 0 .. len(counts) - 1."""
        first = [cache.grow(b, n) for b, n in enumerate(counts)]
        T = sum(counts)
        qs, ks = np.concatenate([[0], np.cumsum(counts)]), np.concatenate([[0], np.cumsum(cache.tokens[:len(counts)])])
        seq = np.repeat(np.arange(len(counts)), counts)
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(first, counts)])
        for layer in range(L):
            x, r0 = draw(T), g.standard_normal((T, d)).astype(np.float32)
            r = torch.from_numpy(r0).cuda()
            attn.prefill(layer, torch.from_numpy(x).cuda(), r, i32(seq), i32(pos), i32(qs), i32(ks), int(ks[-1]), max(counts))
            got = r.cpu().numpy().astype(np.float64) - r0
            for b, n in enumerate(counts):
                part = slice(qs[b], qs[b + 1])
                want, rows[layer, b] = _oracle(host[layer], x[part], pos[part], rows.get((layer, b), []), rope)
                if n:
                    _close(got[part], want, ("chunk", counts, layer, b))

    def step(live):
        """One token of each live sequence, in a batch of all table rows."""
        n = len(cache.ids)
        pos = [cache.grow(b, 1) if b in live else 0 for b in range(n)]
        seq, kv = [b if b in live else -1 for b in range(n)], [p + 1 if b in live else 0 for b, p in enumerate(pos)]
        for layer in range(L):
            x, r0 = draw(n), g.standard_normal((n, d)).astype(np.float32)
            r = torch.from_numpy(r0).cuda()
            attn.decode(layer, torch.from_numpy(x).cuda(), r, i32(seq), i32(pos), i32(kv))
            got = r.cpu().numpy().astype(np.float64) - r0
            for b in range(n):
                if b not in live:
                    assert not got[b].any(), b             # a padding row's residual stays as it was
                    continue
                want, rows[layer, b] = _oracle(host[layer], x[b:b + 1], np.array([pos[b]]), rows[layer, b], rope)
                _close(got[b], want[0], ("step", layer, b, pos[b]))

    assert [cache.start() for _ in range(2)] == [0, 1]
    chunk([37, 16])
    chunk([20, 3])
    new = cache.fork(0)
    for layer in range(L):
        rows[layer, new] = rows[layer, 0].copy()
    step({0, 1, new})
    cache.end(1)
    for layer in range(L):
        del rows[layer, 1]
    assert cache.compact() > 0
    for _ in range(18):                                    # the fork and its origin write on past a page's end
        step({0, new})
    other = cache.start()
    assert other == 1
    chunk([0, 40])
    step({0, 1, new})
    assert int(cache.status) == 0
    third = cache.fork(1)
    with pytest.raises(ValueError):
        cache.start()
    with pytest.raises(ValueError):
        cache.grow(third, most)
    for s in (0, 1, new, third):
        cache.end(s)
    assert cache.pool.available() == 40
    cache.close()
