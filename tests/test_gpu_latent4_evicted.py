"""A 4-bit cache behind an eviction: calls that would take a token's position for its place, and evictions that fail on
their way."""

import numpy as np
import pytest

from tests.test_gpu_attention_chain import DR, _blocks, _spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def test_positions_are_no_places_behind_an_eviction(torch_cuda):
    """Without places a call on an evicted sequence's row is refused and changes nothing. With them it runs, and so do calls
    without on other rows, on that of a sequence that ended, and on that of the next one there."""
    torch, g = torch_cuda, np.random.default_rng(3)
    from paper_2609_18063_amd import latent
    d = 256
    dev, _ = _blocks(torch, d, 1, 5)
    cache = latent.LatentCache(_spec(16), 1, 20, 3, 64, bits=4, weights=True)
    attn = latent.LatentAttention(d, _spec(16), dev, cache, latent.rope_table(200, DR), max_rows=8)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.from_numpy(g.standard_normal((2, d)).astype(np.float16)).cuda()
    r = torch.zeros(2, d, device="cuda")

    def step(form, rows, places):
        """The last token of each of the first rows, once more."""
        live = [cache.ids[s] is not None for s in range(rows)]
        n = [cache.tokens[s] for s in range(rows)]
        seq, slot = i32([s if k else -1 for s, k in enumerate(live)]), i32([max(k - 1, 0) for k in n])
        pos, kw = slot + i32(cache.evicted[:rows]), dict(slot=slot) if places else {}
        if form == "decode":
            attn.decode(0, x[:rows], r[:rows], seq, pos, i32(n), **kw)
        elif all(live):
            attn.prefill(0, x[:rows], r[:rows], seq, pos, i32(list(range(rows + 1))), i32(np.cumsum([0] + n).tolist()), sum(n), 1, **kw)

    def both(rows, places):
        for form in ("decode", "prefill"):
            step(form, rows, places)

    for n in (31, 41):
        cache.grow(cache.start(), n)
    both(2, False)                                         # nothing is evicted yet
    assert cache.evict(35) == [0, 6, 0]
    cache.grow(1, 1)
    was = [t.clone() for t in (cache.pages, cache.sums, r)]
    for form in ("decode", "prefill"):
        with pytest.raises(ValueError):
            step(form, 2, False)
    assert all(torch.equal(a, b) for a, b in zip(was, (cache.pages, cache.sums, r)))
    both(1, False)
    both(2, True)
    cache.end(1)
    both(2, False)
    assert cache.start() == 1
    cache.grow(1, 31)
    both(2, False)
    assert int(cache.status) == 0
    cache.close()


@pytest.mark.parametrize("call", ["evict_select", "latent4_move"])
def test_an_eviction_that_fails_gives_its_pages_back(torch_cuda, monkeypatch, call):
    """Whatever ends it behind the allocation of the new pages: the pool, the sequences, their rows and sums are as before, and
    the same eviction then runs."""
    torch = torch_cuda
    from paper_2609_18063_amd import binding as B, latent
    cache = latent.LatentCache(_spec(16), 2, 20, 2, 128, bits=4, weights=True)
    for n in (100, 50):
        cache.grow(cache.start(), n)
    cache.pages.random_(0, 256)
    cache.sums.uniform_()
    free, state = cache.pool.available(), [list(cache.ids), list(cache.tokens), list(cache.evicted)]
    was = [cache.sums.clone(), cache.table.clone()]

    def fail(*a, **kw):
        raise torch.cuda.OutOfMemoryError("as if")

    with monkeypatch.context() as m:
        m.setattr(B, call, fail)
        with pytest.raises(torch.cuda.OutOfMemoryError):
            cache.evict(40)
    assert cache.pool.available() == free and [cache.ids, cache.tokens, cache.evicted] == state
    assert torch.equal(cache.sums, was[0]) and torch.equal(cache.table, was[1])
    assert cache.evict(40) == [60, 10] and int(cache.status) == 0
    for s in (0, 1):
        cache.end(s)
    assert cache.pool.available() == 20
    cache.close()
