"""moe_linear_int4_lora at the ends of its ranges: every adapter width with tiles, more tiles than a round of workgroups
has, the most inputs, and rows whose small products are far apart in size."""

import numpy as np
import pytest

from oracle import attention as A
from tests.test_gpu_linear import Linear

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _run(torch, lin, x, dtype=None):
    y = torch.full((len(x), lin.out), 7.0, dtype=dtype or torch.float32, device="cuda")
    lin(torch.from_numpy(x).cuda(), y)
    return y.cpu().numpy()


# whole tiles of 128 x 128 beside split ones (525 tiles: 512 and 13 in parts), just whole ones, and ranks above 16
@pytest.mark.parametrize("T,out,inn,r", [(200, 130, 320, 17), (200, 130, 320, 33), (260, 65, 2112, 64), (193, 300, 64, 32),
                                         (2600, 3200, 512, 16), (2048, 4096, 128, 40)])
def test_tiles(torch_cuda, T, out, inn, r):
    g = np.random.default_rng(T + r)
    lin = Linear(torch_cuda, g, out, inn, r)
    x = g.standard_normal((T, inn)).astype(np.float16)
    lin.check(x, _run(torch_cuda, lin, x))


@pytest.mark.parametrize("T", [3, 20, 200])
def test_most_inputs(torch_cuda, T):
    g = np.random.default_rng(T)
    lin = Linear(torch_cuda, g, 40, 32768, 64)
    x = g.standard_normal((T, 32768)).astype(np.float16)
    lin.check(x, _run(torch_cuda, lin, x))


@pytest.mark.parametrize("T", [3, 40, 200])
def test_large_inputs_of_a_group_without_weights(torch_cuda, T):
    """A group whose scales and zeros are 0 under inputs near fp16's largest: it adds nothing, and takes no bits of what
    the other groups add."""
    g = np.random.default_rng(41)
    lin = Linear(torch_cuda, g, 150, 320, 16)
    q, s, z = lin.qsz
    s[:, 2], z[:, 2] = 0, 0
    lin.lora[0][:, 128:192] = 0
    lin.proj, lin.keep = lin.B.upload_projection(lin.qsz, lin.lora, "cuda")
    x = g.standard_normal((T, 320)).astype(np.float16)
    x[:, 128:192] = 60000
    lin.check(x, _run(torch_cuda, lin, x))


@pytest.mark.parametrize("T", [3, 200])
def test_large_adapter_inputs_without_outputs(torch_cuda, T):
    """B = 0, as an adapter starts, under a large A x."""
    g = np.random.default_rng(42)
    lin = Linear(torch_cuda, g, 150, 320, 16, scale=64.0)
    lin.lora = (np.float16(1000) * lin.lora[0], 0 * lin.lora[1])
    lin.proj, lin.keep = lin.B.upload_projection(lin.qsz, lin.lora, "cuda")
    x = g.standard_normal((T, 320)).astype(np.float16)
    lin.check(x, _run(torch_cuda, lin, x))
