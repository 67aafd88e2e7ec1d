"""dsde_distill_* at the ends of their ranges: masks of any size over whole chunks, losses near 0, very many rows; the
fused call against the two it stands for."""
import pytest
import torch

from rows_reference import WEIGHT_TOL
from test_gpu_distill import DT, inputs, near, reference, run_all

pytestmark = pytest.mark.gpu

MASKS = (-1e4, -1e6, -1e9, -1e10, -1e11, -1e12, -1e13, -1e18, -1e20, -1e29, -1e30, -3.3895313892515355e38)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [0.5, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("tail", [False, True])
def test_chunks_of_masked_logits(gpu_lib, tail, T, dtype):
    """A finite mask over whole chunks of 8,192 logits and over a short last one, whose maxima are the mask."""
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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_loss_near_zero(gpu_lib, dtype):
    """A teacher of one token that the student nearly always gives: loss = log1p(rest), as exact as the sum of the rest's
    weights.  A weight e^-x is off by (1.5 x + 1) 2^-23 of itself at most, the sums of eight in fp32 by 3 2^-24, the
    result by 2^-24."""
    V, gaps = 50257, (12.0, 14.0, 16.0, 18.0, 20.0, 22.0, 24.0)
    g = torch.Generator().manual_seed(8)
    s = torch.randn(len(gaps), V, generator=g) - torch.tensor(gaps)[:, None]
    ids = torch.randint(0, V, (len(gaps), 1), generator=g)
    s = s.scatter(1, ids, 0.0).to(DT[dtype])
    want = torch.log1p(s.double().exp().scatter(1, ids, 0.0).sum(1))
    tol = ((1.5 * torch.tensor(gaps).double() + 1) * 2.0 ** -23 + 4 * 2.0 ** -24) * want
    for loss, _ in run_all(gpu_lib, s, ids.int(), torch.zeros(len(gaps), 1), None, 1.0, torch.ones(len(gaps))):
        assert bool(((loss.double() - want).abs() <= tol).all()), loss.double() / want - 1


def test_small_tail_of_the_teacher(gpu_lib):
    """One entry with all but r of the mass: r = 1 - exp(t - lse) keeps its digits, and the loss's terms theirs.  Each
    term is a product of p or r (exact here but for the fp64 functions) and a logarithm of the student's sums."""
    V, N = 9001, 12
    g = torch.Generator().manual_seed(4)
    s = torch.randn(N, V, generator=g) - 14.0
    ids = torch.randint(0, V, (N, 1), generator=g)
    s.scatter_(1, ids, 0.0)
    lse = 2.0 ** -torch.arange(4, 4 + N).float() * (1 + torch.rand(N, generator=g))
    t = torch.zeros(N, 1)
    p = (-lse.double()).exp()
    r = 1 - p
    rest = s.double().exp().scatter(1, ids, 0.0).sum(1)
    log_all = torch.log1p(rest)
    terms = torch.stack([p * -lse.double(), p * log_all, r * r.log(), -r * rest.log(), r * log_all])
    want = terms.sum(0)
    # rest's weights and their sum move log1p(rest) and log(rest); then fp32's rounding
    tol = (WEIGHT_TOL + 4 * 2.0 ** -24) * (p * log_all + r + r * log_all) + 2.0 ** -24 * want.abs()
    for loss, _ in run_all(gpu_lib, s, ids.int(), t, lse, 1.0, torch.ones(N)):
        assert bool(((loss.double() - want).abs() <= tol).all()), (loss.double() - want) / tol


def test_more_rows_than_one_launch_takes(gpu_lib):
    """2^24 rows and more: a launch of 256 threads for each would pass 2^32 threads."""
    N, V, K = (1 << 24) + 5, 8, 1
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24, N - 1]
    g = torch.Generator().manual_seed(3)
    z[rows] = torch.randn(len(rows), V, generator=g).to(torch.bfloat16).cuda()
    ids = torch.full((N, K), 3, dtype=torch.int32, device="cuda")
    t = torch.ones(N, K, device="cuda")
    w = torch.ones(N, device="cuda")
    s = z[rows].cpu()
    want = reference(s, ids[rows].cpu(), t[rows].cpu(), None, 1.0, torch.ones(len(rows)))
    o = gpu_lib.distill_loss(z, ids, t)
    grad = gpu_lib.distill_grad(z, ids, t, o["record"], w)
    f = gpu_lib.distill_step(z, ids, t, w)
    for x, y in ((o["loss"], grad), (f["loss"], f["grad"])):
        near(x[rows].cpu(), y[rows].cpu(), want, torch.ones(len(rows)), 1.0, "bf16")
        plain = torch.ones(N, dtype=torch.bool, device="cuda")
        plain[rows] = False
        # all other rows are equal
        assert bool((x[plain] == x[2]).all()) and bool((y[plain] == y[2]).all())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,V", [("bf16", 7), ("bf16", 30001), ("bf16", 128256), ("fp32", 9), ("fp32", 70001)])
def test_step_is_loss_and_gradient_bit_for_bit(gpu_lib, dtype, V, tail):
    """The fused call runs the kernels of the other two: the same bits, on rows that are neither left out nor flagged."""
    N, T = 64, 1.3
    s, ids, t, lse = inputs(N, V, min(V, 40), dtype, seed=V, T=T)
    z, i, v, l = s.cuda(), ids.cuda(), t.cuda(), lse.cuda() if tail else None
    w = torch.rand(N, generator=torch.Generator().manual_seed(2)).cuda() - 0.5
    f = gpu_lib.distill_step(z, i, v, w, teacher_lse=l, temperature=T)
    o = gpu_lib.distill_loss(z, i, v, teacher_lse=l, temperature=T)
    g = gpu_lib.distill_grad(z, i, v, o["record"], w, temperature=T)
    torch.cuda.synchronize()
    assert torch.equal(f["loss"], o["loss"]) and torch.equal(f["grad"], g)
