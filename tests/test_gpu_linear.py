"""moe_linear_int4_lora against the float64 projection: row counts on both sides of every launch, input and output
sizes that fill no tile, ranks, output types, strides, values at the ends of fp16, infinities and NaN, and replays of
a captured call. Each value is held to the bound that the oracle derives for it."""

import numpy as np
import pytest

from oracle import attention as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    from paper_2609_18063_amd import binding
    binding.lib()
    return torch


def _weights(g, out, inn, r):
    q = g.integers(0, 256, (out, inn // 2)).astype(np.uint8)
    s = (0.02 / np.sqrt(255 / 12) * g.uniform(0.9, 1.1, (out, inn // 64))).astype(np.float16)
    z = (-7.5 * s.astype(np.float64) + 0.005 * g.uniform(-1, 1, s.shape)).astype(np.float16)
    lora = None
    if r:
        lora = (g.normal(0, 1 / r, (r, inn)).astype(np.float16), g.normal(0, 0.01, (out, r)).astype(np.float16))
    return (q, s, z), lora


class Linear:
    def __init__(self, torch, g, out, inn, r, scale=2.0):
        from paper_2609_18063_amd import binding as B
        self.B, self.torch, self.out, self.inn, self.r, self.scale = B, torch, out, inn, r, scale
        self.qsz, self.lora = _weights(g, out, inn, r)
        self.proj, self.keep = B.upload_projection(self.qsz, self.lora, "cuda")

    def workspace(self, T):
        n = self.B.linear_workspace_bytes(self.out, self.inn, self.r, T)
        return self.torch.full((n,), 255, dtype=self.torch.uint8, device="cuda")

    def __call__(self, x, y, add=False, ws=None):
        self.B.linear_int4(self.proj, self.out, self.inn, self.r, self.scale, x, y,
                           self.workspace(x.shape[0]) if ws is None else ws, add=add)

    def check(self, x, got, f16=False, base=None):
        y, mag = A.projection(self.qsz, self.lora, self.scale, x)
        bound = A.projection_bound(y, mag, self.inn, self.r, f16)
        if base is not None:
            y = y + base
            bound = bound + A.SINGLE * np.abs(y)
        off = np.abs(got.astype(np.float64) - y) - bound
        assert np.isfinite(got).all() and (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))


SHAPES = [(1, 64, 64, 0), (1, 17, 128, 3), (1, 576, 2048, 16), (2, 100, 192, 1), (13, 33, 576, 16), (15, 1, 4096, 8),
          (16, 16, 64, 64), (16, 513, 8192, 16), (17, 48, 320, 17), (33, 65, 2048, 0), (48, 130, 704, 33), (64, 31, 1024, 16),
          (65, 127, 64, 0), (65, 129, 128, 16), (100, 5001, 2048, 16), (127, 64, 4096, 64), (128, 128, 448, 7), (129, 1, 512, 2),
          (300, 300, 8192, 16), (513, 200, 2112, 0)]


@pytest.mark.parametrize("T,out,inn,r", SHAPES)
def test_types(torch_cuda, T, out, inn, r):
    torch, g = torch_cuda, np.random.default_rng(T * 7 + out)
    lin = Linear(torch, g, out, inn, r)
    x = g.standard_normal((T, inn)).astype(np.float16)
    xt = torch.from_numpy(x).cuda()
    for dtype in (torch.float32, torch.float16):
        y = torch.full((T, out), 7.0, dtype=dtype, device="cuda")
        lin(xt, y)
        lin.check(x, y.cpu().numpy(), dtype == torch.float16)
    base = g.standard_normal((T, out)).astype(np.float32)
    y = torch.from_numpy(base).cuda()
    lin(xt, y, add=True)
    lin.check(x, y.cpu().numpy(), base=base.astype(np.float64))


@pytest.mark.parametrize("T,out,inn,r", [(3, 40, 128, 4), (40, 70, 192, 16), (150, 131, 320, 9)])
def test_strides_leave_the_rest(torch_cuda, T, out, inn, r):
    torch, g = torch_cuda, np.random.default_rng(5)
    lin = Linear(torch, g, out, inn, r)
    x = g.standard_normal((T, inn)).astype(np.float16)
    wide = torch.full((T, inn + 24), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :inn] = torch.from_numpy(x).cuda()
    for dtype in (torch.float32, torch.float16):
        y = torch.full((T + 2, out + 5), 7.0, dtype=dtype, device="cuda")
        lin(wide[:, :inn], y[:T, :out])
        got = y.cpu().numpy()
        lin.check(x, got[:T, :out], dtype == torch.float16)
        assert (got[T:] == 7).all() and (got[:, out:] == 7).all()


@pytest.mark.parametrize("T", [1, 20, 90])
@pytest.mark.parametrize("size", [6e4, 1e-4, 6e-8])
def test_ends_of_fp16(torch_cuda, T, size):
    """Activations near fp16's largest and among its subnormals: the sums stay fp32's."""
    torch, g = torch_cuda, np.random.default_rng(6)
    lin = Linear(torch, g, 50, 256, 16)
    x = (g.uniform(-1, 1, (T, 256)) * size).astype(np.float16)
    x[0] = np.float16(size)                      # group sums beyond fp16 where size is its end
    y = torch.empty(T, 50, dtype=torch.float32, device="cuda")
    lin(torch.from_numpy(x).cuda(), y)
    lin.check(x, y.cpu().numpy())


@pytest.mark.parametrize("T", [5, 16, 40, 200])
def test_nonfinite_rows_stay_alone(torch_cuda, T):
    torch, g = torch_cuda, np.random.default_rng(7)
    lin = Linear(torch, g, 70, 320, 16)
    x = g.standard_normal((T, 320)).astype(np.float16)
    bad = sorted({1, T // 2, T - 1})
    p = x.copy()
    for k, t in enumerate(bad):
        p[t, 3 + k] = (np.inf, -np.inf, np.nan)[k % 3]
    out = []
    for v in (x, p):
        y = torch.empty(T, 70, dtype=torch.float32, device="cuda")
        lin(torch.from_numpy(v).cuda(), y)
        out.append(y.cpu().numpy())
    good = np.setdiff1d(np.arange(T), bad)
    assert np.array_equal(out[0][good], out[1][good]) and not np.isfinite(out[1][bad]).any()


def test_zero_rows_and_one_row_of_many(torch_cuda):
    torch, g = torch_cuda, np.random.default_rng(8)
    lin = Linear(torch, g, 60, 256, 16)
    y = torch.full((0, 60), 7.0, device="cuda")
    lin(torch.empty(0, 256, dtype=torch.float16, device="cuda"), y, ws=lin.workspace(1))
    x = g.standard_normal((90, 256)).astype(np.float16)
    x[:] = x[0]                                  # the same row everywhere gives the same row everywhere
    y = torch.empty(90, 60, device="cuda")
    lin(torch.from_numpy(x).cuda(), y)
    assert (y == y[0]).all()


@pytest.mark.parametrize("T", [1, 30, 100])
def test_graph_replays_on_a_side_stream(torch_cuda, T):
    torch, g = torch_cuda, np.random.default_rng(9)
    lin = Linear(torch, g, 200, 1024, 16)
    x = torch.zeros(T, 1024, dtype=torch.float16, device="cuda")
    y, ws = torch.empty(T, 200, device="cuda"), lin.workspace(T)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        lin(x, y, ws=ws)
    for k in range(4):
        v = g.standard_normal((T, 1024)).astype(np.float16)
        x.copy_(torch.from_numpy(v))
        graph.replay()
        got = y.clone()
        lin(x, y, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(got, y), k
        lin.check(v, got.cpu().numpy())


# Either side of the rule for tiles (more than 192 rows, or workgroups of 32 x 32 beyond the CUs), and what the
# calls above check of few rows.
@pytest.mark.parametrize("T,out,inn,r", [(192, 65, 2048, 16), (193, 65, 2048, 16), (20, 8200, 128, 3), (33, 4097, 2112, 5),
                                         (64, 8193, 64, 0), (40, 8193, 2048, 16), (256, 129, 192, 1)])
def test_types_around_the_tiles(torch_cuda, T, out, inn, r):
    test_types(torch_cuda, T, out, inn, r)


def test_strides_leave_the_rest_with_tiles(torch_cuda):
    test_strides_leave_the_rest(torch_cuda, 210, 131, 320, 9)


@pytest.mark.parametrize("size", [6e4, 1e-4, 6e-8])
def test_ends_of_fp16_with_tiles(torch_cuda, size):
    test_ends_of_fp16(torch_cuda, 195, size)


def test_graph_replays_with_tiles(torch_cuda):
    test_graph_replays_on_a_side_stream(torch_cuda, 230)
