"""dsde_distill_* against their definition in 64 bits and against differences."""
import math

import pytest
import torch

from rows_reference import distill_row

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def inputs(N, V, K, dtype, seed=0, T=1.0, sigma=0.7):
    """Student, teacher entries and log-normaliser (CPU)."""
    g = torch.Generator().manual_seed(seed)
    t = 3.0 * torch.randn(N, V, generator=g)
    s = (t + sigma * torch.randn(N, V, generator=g)).to(DT[dtype])
    v, ids = t.topk(min(K, V), dim=1)
    if K > V:
        pad = (0, K - V)
        v, ids = torch.nn.functional.pad(v, pad, value=5.0), torch.nn.functional.pad(ids, pad, value=-1)
    return s, ids.int(), v, torch.logsumexp(t.double() / T, 1).float()


def reference(s, ids, t, lse, T, weight):
    loss, grad = [], []
    for i in range(len(s)):
        a, b = distill_row(s[i].float(), ids[i], t[i], None if lse is None else lse[i], T)
        loss.append(a)
        grad.append(b * float(weight[i]))
    return torch.stack(loss), torch.stack(grad)


def near(loss, grad, want, weight, T, dtype):
    """Loss: logarithms of sums that are good to a few 1e-7, rounded to fp32.  Gradient: a
    difference of probabilities that are good to 4e-6 of themselves (the sampling
    tests derive it), rounded to the logits' type."""
    wl, wg = want
    assert float((loss.double() - wl).abs().max()) <= 2e-6 + 2e-7 * float(wl.abs().max())
    scale = (weight.double().abs() / T)[:, None]
    rounding = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24  # half a unit in the last of 8 and of 24 places
    bound = scale * 8e-6 + wg.abs() * (rounding * 1.01 + 8e-6)
    assert bool(((grad.double() - wg).abs() <= bound).all())


def run_all(lib, s, ids, t, lse, T, weight):
    """Loss and gradient by the two calls, by the fused one and by autograd: (loss, grad) each, on the CPU."""
    z, i, v = s.cuda(), ids.cuda(), t.cuda()
    l, w = None if lse is None else lse.cuda(), weight.cuda()
    o = lib.distill_loss(z, i, v, teacher_lse=l, temperature=T)
    assert (o["row_err"] == 0).all()
    g = lib.distill_grad(z, i, v, o["record"], w, temperature=T)
    f = lib.distill_step(z, i, v, w, teacher_lse=l, temperature=T)
    assert (f["row_err"] == 0).all()
    x = z.clone().requires_grad_(True)
    a = lib.distill(x, i, v, teacher_lse=l, temperature=T)
    (a * w).sum().backward()
    torch.cuda.synchronize()
    return [(o["loss"].cpu(), g.cpu()), (f["loss"].cpu(), f["grad"].cpu()), (a.detach().cpu(), x.grad.cpu())]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,K,T", [(1, 1, 1.0), (2, 1, 1.0), (7, 3, 2.0), (8, 8, 1.0), (9, 12, 1.5), (65, 33, 0.5),
                                   (1000, 256, 1.0), (8191, 16, 1.0), (8192, 64, 2.0), (8193, 1, 1.0),
                                   (50257, 100, 1.5), (140001, 64, 1.0)])
def test_loss_and_gradient(gpu_lib, V, K, T, tail, dtype):
    s, ids, t, lse = inputs(5, V, K, dtype, seed=V + K, T=T)
    lse = lse if tail else None
    weight = torch.tensor([1.0, 0.25, -3.0, 1e-4, 7.0])
    want = reference(s, ids, t, lse, T, weight)
    for loss, grad in run_all(gpu_lib, s, ids, t, lse, T, weight):
        near(loss, grad, want, weight, T, dtype)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(gpu_lib, tail):
    """Central differences of the loss along random directions: their error is h^2 / 6 times a third
    derivative of order one, and the losses' rounding, 1e-6, over h."""
    N, V, K, T, h = 6, 3000, 40, 1.5, 0.01
    s, ids, t, lse = inputs(N, V, K, "fp32", seed=2, T=T)
    lse = lse.cuda() if tail else None
    z, i, v = s.cuda(), ids.cuda(), t.cuda()
    g = gpu_lib.distill_step(z, i, v, torch.ones(N, device="cuda"), teacher_lse=lse, temperature=T)["grad"]
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        d = torch.randn(N, V, generator=gen, device="cuda")
        up, down = (gpu_lib.distill_loss(z + e * d, i, v, teacher_lse=lse, temperature=T)["loss"] for e in (h, -h))
        got = (up - down).double() / (2 * h)
        assert float((got - (g * d).double().sum(1)).abs().max()) <= 1e-4 + 2e-6 / h


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [False, True])
def test_unused_entries_and_masks(gpu_lib, tail, dtype):
    """Entries of id -1 and of -inf, rows without any, student masks outside the entries (both kinds),
    a teacher whose entries hold all its mass."""
    V, K, T = 10001, 20, 1.0
    s, ids, t, lse = inputs(7, V, K, "fp32", seed=4)
    ids[0, ::2] = -1
    ids[1] = -1
    t[2, 3:] = -math.inf
    t[3] = -math.inf
    keep = torch.zeros(V, dtype=torch.bool)
    keep[ids[4].long()] = True
    s[4][~keep] = -math.inf
    s[5][~torch.zeros(V, dtype=torch.bool).index_fill(0, ids[5].long(), True)] = -3.3895313892515355e38
    lse[6] = torch.logsumexp(t[6].double(), 0).float()
    s = s.to(DT[dtype])
    lse = lse if tail else None
    weight = torch.ones(7)
    if tail:  # the tail of row 5 lies where the student's logits are the lowest value: its loss is not a small number
        lse[5] = torch.logsumexp(t[5].double(), 0).float() + 1e-3
    want = reference(s, ids, t, lse, T, weight)
    rows = [i for i in range(7) if not (tail and i == 5)]
    for loss, grad in run_all(gpu_lib, s, ids, t, lse, T, weight):
        near(loss[rows], grad[rows], (want[0][rows], want[1][rows]), weight[rows], T, dtype)
        assert bool(torch.isfinite(grad).all())
        if not tail:
            assert float(loss[1]) == 0.0 and bool((grad[1] == 0).all())


def test_a_student_that_agrees(gpu_lib):
    """Student and teacher equal: a loss and a gradient of rounding's size, also in a tail of 1e-5."""
    N, V, K = 4, 20000, 64
    g = torch.Generator().manual_seed(7)
    t = 4.0 * torch.randn(N, V, generator=g)
    t[:, :8] += 14.0
    v, ids = t.topk(K, dim=1)
    lse = torch.logsumexp(t.double(), 1).float()
    for loss, grad in run_all(gpu_lib, t, ids.int(), v, lse, 1.0, torch.ones(N)):
        assert float(loss.abs().max()) <= 4e-6 and float(grad.abs().max()) <= 8e-6


def test_data_errors_flag_their_row_alone(gpu_lib):
    N, V, K = 10, 9000, 6
    s, ids, t, lse = inputs(N, V, K, "fp32", seed=1)
    ids[0, 2] = V
    ids[1, 2] = -2
    ids[2, 5] = ids[2, 0]
    s[3, 8999] = math.nan
    s[4, 0] = math.inf
    t[5, 0] = math.nan
    t[6, 1] = math.inf
    lse[7] = math.inf
    s[8, ids[8, 0].long()] = -math.inf
    e = gpu_lib
    want = [e.ERR_TOKEN] * 3 + [e.ERR_LOGIT] * 6 + [0]
    ref = reference(s[9:], ids[9:], t[9:], lse[9:], 1.0, torch.ones(1))
    z, i, v, l = s.cuda(), ids.cuda(), t.cuda(), lse.cuda()
    o = e.distill_loss(z, i, v, teacher_lse=l)
    assert o["row_err"].tolist() == want and o["loss"][:9].isnan().all()
    grad = e.distill_grad(z, i, v, o["record"], torch.ones(N, device="cuda"))
    f = e.distill_step(z, i, v, torch.ones(N, device="cuda"), teacher_lse=l)
    assert f["row_err"].tolist() == want and f["loss"][:9].isnan().all()
    for loss, g in ((o["loss"], grad), (f["loss"], f["grad"])):
        assert (g[:9] == 0).all()
        near(loss[9:].cpu(), g[9:].cpu(), ref, torch.ones(1), 1.0, "fp32")


@pytest.mark.parametrize("N,V", [(40, 9001), (700, 4099), (300, 33000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_step_leaves_out_rows_of_weight_zero(gpu_lib, N, V, dtype):
    """Padding rows: nothing of theirs is read or checked; the others as without them."""
    s, ids, t, lse = inputs(N, V, 9, dtype, seed=N)
    weight = torch.rand(N, generator=torch.Generator().manual_seed(1)) + 0.1
    z, i, v, l, w = s.cuda(), ids.cuda(), t.cuda(), lse.cuda(), weight.cuda()
    full = gpu_lib.distill_step(z, i, v, w, teacher_lse=l)
    z2, i2, w2 = z.clone(), i.clone(), w.clone()
    z2[::3] = math.nan
    i2[::3] = -9
    w2[::3] = 0.0
    part = gpu_lib.distill_step(z2, i2, v, w2, teacher_lse=l)
    assert (part["row_err"] == 0).all()
    out = torch.arange(N) % 3 == 0
    for k in ("loss", "grad"):
        assert (part[k][out.cuda()] == 0).all()
        assert torch.equal(part[k][~out.cuda()], full[k][~out.cuda()]), k


@pytest.mark.parametrize("N,V", [(5, 8200), (600, 5001), (260, 40000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place_strided_and_repeated(gpu_lib, N, V, dtype):
    """Slices of wider rows, the gradient over the logits, another stream: the same bits."""
    s, ids, t, lse = inputs(N, V, 16, dtype, seed=V)
    wide = torch.zeros(N, V + 21, dtype=DT[dtype], device="cuda")
    wide[:, 3:3 + V] = s.cuda()
    i, v, l, w = ids.cuda(), t.cuda(), lse.cuda(), torch.rand(N, device="cuda") + 0.5
    ref = gpu_lib.distill_step(s.cuda(), i, v, w, teacher_lse=l)
    z = wide[:, 3:3 + V]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for kw in ({}, dict(stream=side), dict(grad=torch.empty_like(wide)[:, 1:1 + V])):
        got = gpu_lib.distill_step(z, i, v, w, teacher_lse=l, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got["loss"], ref["loss"]) and torch.equal(got["grad"], ref["grad"])
    edge = (wide[:, :3].clone(), wide[:, 3 + V:].clone())
    o = gpu_lib.distill_loss(z, i, v, teacher_lse=l)
    two = wide.clone()[:, 3:3 + V]
    gpu_lib.distill_grad(two, i, v, o["record"], w, grad=two)
    gpu_lib.distill_step(z, i, v, w, teacher_lse=l, grad=z)
    assert torch.equal(z, ref["grad"]) and torch.equal(two, ref["grad"])
    assert torch.equal(wide[:, :3], edge[0]) and torch.equal(wide[:, 3 + V:], edge[1])


@pytest.mark.parametrize("dtype,V", [("bf16", 7), ("bf16", 30000), ("bf16", 50257), ("bf16", 70001), ("bf16", 128256),
                                     ("bf16", 152064), ("bf16", 160001), ("fp32", 9), ("fp32", 40001),
                                     ("fp32", 65536), ("fp32", 70001), ("fp32", 128256)])
def test_step_of_many_rows(gpu_lib, dtype, V):
    """The one-pass form of the fused call, at every width of it and beyond, against the definition."""
    N, K, T = 300, min(V, 40), 1.3
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (3.0 * torch.randn(N, V, generator=g, device="cuda")).to(DT[dtype])
    t = (z.float() + torch.randn(N, V, generator=g, device="cuda")).to(DT[dtype]).float()
    v, ids = t.topk(K, dim=1)
    ids = ids.int()
    ids[5, ::2] = -1
    ids[6] = -1
    ids[7, 0] = V
    lse = torch.logsumexp(t.double() / T, 1).float()
    w = torch.rand(N, generator=g, device="cuda") + 0.1
    w[8] = 0.0
    for l in (lse, None):
        o = gpu_lib.distill_step(z, ids, v, w, teacher_lse=l, temperature=T)
        two = gpu_lib.distill_loss(z, ids, v, teacher_lse=l, temperature=T)
        torch.cuda.synchronize()
        rows = [0, 5, 6, 9, 100, 299]
        want = reference(z[rows].cpu(), ids[rows].cpu(), v[rows].cpu(), None if l is None else l[rows].cpu(), T,
                         w[rows].cpu())
        near(o["loss"][rows].cpu(), o["grad"][rows].cpu(), want, w[rows].cpu(), T, dtype)
        assert int(o["row_err"][7]) == gpu_lib.ERR_TOKEN and bool(o["loss"][7].isnan()) and bool((o["grad"][7] == 0).all())
        assert float(o["loss"][8]) == 0.0 and bool((o["grad"][8] == 0).all())
        keep = torch.ones(N, dtype=torch.bool, device="cuda")
        keep[7:9] = False
        assert float((o["loss"] - two["loss"])[keep].abs().max()) <= 4e-6


def test_graph_replays(gpu_lib):
    N, V, K = 300, 9000, 12
    s, ids, t, lse = inputs(N, V, K, "bf16", seed=3)
    z, i, v, l = s.cuda(), ids.cuda(), t.cuda(), lse.cuda()
    w = torch.ones(N, device="cuda")
    ws = gpu_lib.new_distill_workspace(N, V)
    grad = torch.empty_like(z)
    out = gpu_lib.distill_step(z, i, v, w, teacher_lse=l, grad=grad, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu_lib.distill_step(z, i, v, w, teacher_lse=l, grad=grad, out=out, workspace=ws)
    for step in range(4):
        z.normal_(0.0, 2.0, generator=torch.Generator(device="cuda").manual_seed(step))
        want = gpu_lib.distill_step(z, i, v, w, teacher_lse=l)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["loss"], want["loss"]) and torch.equal(grad, want["grad"])


def test_no_rows(gpu_lib):
    z = torch.empty(0, 100, device="cuda")
    ids, t = torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda")
    assert gpu_lib.distill_step(z, ids, t, torch.empty(0, device="cuda"))["grad"].shape == (0, 100)
    assert gpu_lib.distill_loss(z, ids, t)["loss"].numel() == 0


def test_offsets_beyond_32_bits(gpu_lib):
    """More than 2^31 logits and 2^32 bytes."""
    N, V, K = 34000, 65536, 4
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(K, dtype=torch.int32, device="cuda").expand(N, K).contiguous()
    t = torch.ones(N, K, device="cuda")
    rows = [0, 32767, 33999]
    g = torch.Generator().manual_seed(3)
    for i in rows:
        z[i] = torch.randn(V, generator=g).to(torch.bfloat16).cuda()
    s = z[rows].cpu()
    w = torch.ones(N, device="cuda")
    o = gpu_lib.distill_step(z, ids, t, w, grad=z)
    want = reference(s, ids[rows].cpu(), t[rows].cpu(), None, 1.0, torch.ones(3))
    near(o["loss"][rows].cpu(), z[rows].cpu(), want, torch.ones(3), 1.0, "bf16")
