"""dsde_distill_* at the ends of their ranges: masks of any size over whole chunks."""
import pytest
import torch

from test_gpu_distill import DT, inputs, near, reference, run_all

pytestmark = pytest.mark.gpu

MASKS = (-1e4, -1e6, -1e9, -1e10, -1e11, -1e12, -1e13, -1e18, -1e20, -1e29, -1e30, -3.3895313892515355e38)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [0.5, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("tail", [False, True])
def test_chunks_of_masked_logits(gpu_lib, tail, T, dtype):
    """A finite mask over whole chunks of 8,192 logits and over a short last one: the chunks' own maxima are the mask."""
    V, K = 3 * 8192 + 700, 24
    s, _, t, _ = inputs(len(MASKS), V, K, "fp32", seed=9)
    out = torch.zeros(V, dtype=torch.bool)
    out[8192:16384] = True
    out[3 * 8192:] = True
    for row, mask in zip(s, MASKS):
        row[out] = mask
    s = s.to(DT[dtype])
    wide = s.float() + 0.5 * torch.randn(s.shape, generator=torch.Generator().manual_seed(1))
    t, ids = wide.masked_fill(out, -1e5).topk(K, dim=1)
    lse = torch.logsumexp(wide.masked_fill(out, -float("inf")).double() / T, 1).float() if tail else None
    weight = torch.linspace(0.5, 2.0, len(MASKS))
    want = reference(s, ids.int(), t, lse, T, weight)
    for loss, grad in run_all(gpu_lib, s, ids.int(), t, lse, T, weight):
        near(loss, grad, want, weight, T, dtype)


@pytest.mark.parametrize("base", [2.0 ** 20, -(2.0 ** 20), 2.0 ** 19.99, -(2.0 ** 22)])
@pytest.mark.parametrize("tail", [False, True])
def test_chunks_on_both_sides_of_a_large_offset(gpu_lib, tail, base):
    """Rows far from 0 whose chunks' largest logits lie on both sides of 2^20 ln 2, beyond which a chunk's exponents are
    taken from differences."""
    V, K, N = 5 * 8192 + 11, 24, 8
    g = torch.Generator().manual_seed(3)
    t = 2.0 * torch.randn(N, V, generator=g)
    s = t + 0.5 * torch.randn(N, V, generator=g)
    s = (s.double() + base * 0.6931471805599453 - 6.0).float()  # fp32's spacing there is a sixteenth
    v, ids = t.topk(K, dim=1)
    lse = torch.logsumexp(t.double(), 1).float() if tail else None
    want = reference(s, ids.int(), v, lse, 1.0, torch.ones(N))
    for loss, grad in run_all(gpu_lib, s, ids.int(), v, lse, 1.0, torch.ones(N)):
        near(loss, grad, want, torch.ones(N), 1.0, "fp32")
