"""The largest calls that the 4-bit cache's prompt form takes with sums, without a GPU (the workspace is too small for each, so
that none is enqueued)."""

import ctypes

import pytest

from tests.test_attention_abi_cpu import P, _cache, _spec


@pytest.fixture(scope="module")
def B():
    from paper_2609_18063_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("heads,n", [(128, 60000), (128, 1), (127, 65536)])
def test_sums_launches_are_in_range(B, heads, n):
    """The sums' launch, 512 threads for each head and 128 tokens and one such tile more a sequence, stays under 2^32; with
    more the call is refused before anything of it runs. Without sums there is no such launch."""
    most = ((1 << 32) - 1) // (heads * 512) * 128 + 127 - n * 128

    def call(kv, sums):
        spec, cache = _spec(B, heads=heads), _cache(B, n_seqs=n)
        return B.lib().moe_latent4_prefill(ctypes.byref(spec), ctypes.byref(cache), P[2], P[3], n, P[4], P[5], n, kv, 1, P[6],
                                           P[9] if sums else None, 30, 30, P[7], P[8], 16, None)
    assert call(most, True) == B.MOE_ENOMEM
    assert call(most + 1, True) == B.MOE_EINVAL
    assert call(most + 1, False) == B.MOE_ENOMEM
