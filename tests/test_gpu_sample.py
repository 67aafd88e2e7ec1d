"""dsde_sample against its definition in 64 bits."""
import math

import pytest
import torch

from rows_reference import check_draw, sample_row

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (temperature, top_k, top_p, min_p)
FILTERS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 5, 1.0, 0.0), (1.0, 300, 0.8, 0.0), (1.3, 0, 1.0, 0.02),
           (0.0, 3, 0.5, 0.9), (1.0, 2000, 1.0, 0.0), (1.5, 0, 0.999, 0.0), (2.0, 3000, 0.97, 0.001), (1.0, 1, 1.0, 0.0),
           (0.05, 0, 0.5, 0.0), (4.0, 0, 1.0, 1e-4)]


def draw(lib, z, par, u, **kw):
    R = len(u)
    dev = "cuda"
    f32 = dict(dtype=torch.float32, device=dev)
    T, k, p, m = (list(x) for x in zip(*par))
    o = lib.sample(z.to(dev) if z.device.type == "cpu" else z, torch.tensor(T, **f32), torch.as_tensor(u, **f32),
                   top_k=torch.tensor(k, dtype=torch.int32, device=dev), top_p=torch.tensor(p, **f32),
                   min_p=torch.tensor(m, **f32), kept=True, **kw)
    torch.cuda.synchronize()
    assert o["tokens"].shape == (R,)
    return {k: v.cpu() for k, v in o.items()}


def check(lib, z, par, u, **kw):
    """Every row of z (CPU) against the definition."""
    o = draw(lib, z, par, u, **kw)
    for i, (T, k, p, m) in enumerate(par):
        assert int(o["row_err"][i]) == 0, i
        # settings as the call gets them
        T, p, m = (float(torch.tensor(x, dtype=torch.float32)) for x in (T, p, m))
        check_draw(z[i].float(), T, k, p, m, float(torch.tensor(u[i], dtype=torch.float32)), int(o["tokens"][i]),
                   float(o["logprob"][i]), int(o["kept"][i]))
    return o


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 15, 64, 65, 511, 513, 1025, 8191, 8192, 8193, 32000, 50257, 70001])
def test_draws_follow_the_definition(gpu_lib, V, dtype):
    g = torch.Generator().manual_seed(V)
    R = 2 * len(FILTERS)
    z = (4.0 * torch.randn(R, V, generator=g)).to(DT[dtype])
    check(gpu_lib, z, FILTERS * 2, torch.rand(R, generator=g).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("par", [(1.0, 0, 1.0, 0.0), (1.0, 40, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05),
                                 (1.0, 1500, 0.95, 0.0), (1.2, 0, 0.99, 0.0)])
def test_a_grid_of_uniforms(gpu_lib, par, dtype):
    """The whole inverse CDF of one row, its ends among them."""
    g = torch.Generator().manual_seed(3)
    u = [0.0, 2 ** -24, 1 - 2 ** -24] + [i / 61 for i in range(61)]
    z = (3.0 * torch.randn(1, 20000, generator=g)).to(DT[dtype]).expand(len(u), -1).contiguous()
    check(gpu_lib, z, [par] * len(u), u)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [5, 600, 3000, 40000])
def test_equal_logits_rank_by_id(gpu_lib, V, dtype):
    """A constant row: every filter keeps the lowest ids (more of them than the select
    kernel sorts at once, in the wide rows), and +0 and -0 are equal."""
    par = [(1.0, k, p, 0.0) for k in (0, 1, 4, 700, 2500) for p in (1.0, 0.37)] + [(1.0, 0, 1.0, 1.0), (0.0, 0, 1.0, 0.0)]
    u = [(0.999 * i / len(par)) for i in range(len(par))]
    for value in (0.0, 2.5, -7.0, -3.3895313892515355e38):
        z = torch.full((len(par), V), value).to(DT[dtype])
        if value == 0.0:
            z[:, 1::2] = -0.0
        o = check(gpu_lib, z, par, u)
        for i, (_, k, p, _) in enumerate(par):
            if k and p == 1.0:
                assert int(o["kept"][i]) == min(k, V)
        assert int(o["tokens"][-1]) == 0 and int(o["kept"][-1]) == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mask", [-math.inf, -3.3895313892515355e38, -1e30, -65504.0])
def test_masked_tokens(gpu_lib, mask, dtype):
    """Rows whose mask leaves one token, a few, or many, at either end and in the middle."""
    g = torch.Generator().manual_seed(11)
    V = 30011
    z = torch.full((len(FILTERS) * 3, V), mask)
    for i in range(len(z)):
        n = (1, 9, 6000)[i // len(FILTERS)]
        first = (0, V - n, V // 2)[i % 3]
        z[i, first:first + n] = 2.0 * torch.randn(n, generator=g)
    check(gpu_lib, z.to(DT[dtype]), FILTERS * 3, torch.rand(len(z), generator=g).tolist())


def test_peaked_and_shifted_rows(gpu_lib):
    """One logit far above the others, large offsets of the whole row, and small differences."""
    g = torch.Generator().manual_seed(5)
    V = 12345
    rows = []
    for i in range(len(FILTERS)):
        z = torch.randn(V, generator=g) * (0.01 if i % 3 == 0 else 1.0)
        z += (0.0, 1e4, -1e4, 3e-3)[i % 4]
        if i % 2:
            z[(7 * i) % V] += 60.0
        rows.append(z)
    check(gpu_lib, torch.stack(rows), FILTERS, torch.rand(len(rows), generator=g).tolist())


def test_a_wide_vocabulary(gpu_lib):
    g = torch.Generator().manual_seed(6)
    z = (2.0 * torch.randn(6, 1 << 20, generator=g)).to(torch.bfloat16)
    par = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (1.0, 9000, 1.0, 0.0),
           (0.0, 0, 1.0, 0.0)]
    check(gpu_lib, z, par, torch.rand(6, generator=g).tolist())


def test_data_errors_flag_their_row_alone(gpu_lib):
    V = 9000
    z = torch.randn(12, V, generator=torch.Generator().manual_seed(1))
    z[0, 8500] = math.nan
    z[1, 3] = math.inf
    z[2] = -math.inf
    par = [(1.0, 0, 1.0, 0.0), (1.0, 9, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (1e6, 0, 1.0, 0.0),
           (math.nan, 0, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.5, 0.0), (1.0, 0, 1.0, 1.5), (1.0, 0, math.nan, 0.0),
           (1.0, 0, 1.0, 0.0), (1.0, -4, 1.0, 0.0)]
    u = [0.5] * 10 + [1.0, 0.5]
    o = draw(gpu_lib, z, par, u, pad_id=-7)
    e = gpu_lib
    want = [e.ERR_LOGIT] * 3 + [e.ERR_TEMP] * 3 + [e.ERR_FILTER] * 4 + [e.ERR_UNIFORM, 0]
    assert o["row_err"].tolist() == want
    assert o["tokens"][:11].tolist() == [-7] * 11 and o["kept"][:11].tolist() == [0] * 11
    assert o["logprob"][:11].isnan().all()
    check_draw(z[11], 1.0, 0, 1.0, 0.0, 0.5, int(o["tokens"][11]), float(o["logprob"][11]), int(o["kept"][11]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strided_rows_streams_and_repeats(gpu_lib, dtype):
    """Slices of wider rows on another stream, buffers reused: the same bits as contiguous rows."""
    g = torch.Generator().manual_seed(8)
    R, V = len(FILTERS), 10007
    wide = (4.0 * torch.randn(R, V + 22, generator=g)).to(DT[dtype]).cuda()
    u = torch.rand(R, generator=g).tolist()
    ref = draw(gpu_lib, wide[:, 3:3 + V].contiguous(), FILTERS, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = gpu_lib.new_sample_workspace(2 * R, V + 5)
    ws.fill_(0xff)
    torch.cuda.synchronize()
    for kw in ({}, dict(stream=side), dict(workspace=ws), dict(workspace=ws)):
        got = draw(gpu_lib, wide[:, 3:3 + V], FILTERS, u, **kw)
        for k in ref:
            assert torch.equal(got[k], ref[k]), k
    assert gpu_lib.sample(wide[:0], torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))["tokens"].numel() == 0


def test_graph_replays(gpu_lib):
    """Captured once, replayed over changing inputs with eager work between the replays."""
    R, V = 7, 33000
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.empty(R, V, device="cuda", dtype=torch.bfloat16)
    u = torch.empty(R, device="cuda")
    T = torch.ones(R, device="cuda")
    k = torch.tensor([0, 5, 0, 3000, 0, 100, 0], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 1.0, 0.9, 0.9, 0.99, 0.5, 1.0], device="cuda")
    ws = gpu_lib.new_sample_workspace(R, V)
    z.normal_(0.0, 3.0, generator=g)
    u.uniform_(generator=g)
    out = gpu_lib.sample(z, T, u, top_k=k, top_p=p, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu_lib.sample(z, T, u, top_k=k, top_p=p, out=out, workspace=ws)
    for _ in range(4):
        z.normal_(0.0, 3.0, generator=g)
        u.uniform_(generator=g)
        want = gpu_lib.sample(z, T, u, top_k=k, top_p=p)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["tokens"], want["tokens"]) and torch.equal(out["logprob"], want["logprob"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_greedy_rows_without_filters(gpu_lib, dtype):
    """T = 0 with no filter array at all: the lowest of very many equal maxima, and ordinary rows beside."""
    V = 50000
    z = torch.randn(6, V, generator=torch.Generator().manual_seed(2))
    z[0] = 1.5
    z[1] = -3.3895313892515355e38
    z[2, 100:] = 9.0
    z[3, ::2] = -math.inf
    z = z.to(DT[dtype])
    T = torch.tensor([0.0, 0.0, 0.0, 0.0, 1.0, 0.0])
    o = gpu_lib.sample(z.cuda(), T.cuda(), torch.full((6,), 0.5, device="cuda"), kept=True)
    for i in (0, 1, 2, 3, 5):
        best = int((z[i].float() == z[i].float().max()).int().argmax())
        assert int(o["tokens"][i]) == best and int(o["kept"][i]) == 1 and int(o["row_err"][i]) == 0
    check_draw(z[4].float(), 1.0, 0, 1.0, 0.0, 0.5, int(o["tokens"][4]), float(o["logprob"][4]), int(o["kept"][4]))


def test_frequencies(gpu_lib):
    """Draws under top-k and top-p over many uniforms have the kept tokens' probabilities."""
    g = torch.Generator().manual_seed(4)
    R, V = 4096, 4000
    z = (3.0 * torch.randn(1, V, generator=g)).expand(R, V).contiguous()
    u = ((torch.arange(R) + 0.5) / R).tolist()
    o = draw(gpu_lib, z, [(1.0, 30, 0.9, 0.0)] * R, u)
    ids, e, lo, hi = sample_row(z[0], 1.0, 30, float(torch.tensor(0.9)), 0.0)
    assert lo == hi
    n = torch.bincount(o["tokens"], minlength=V).double()
    w = torch.zeros(V, dtype=torch.float64)
    w[ids[:lo]] = e[:lo] / e[:lo].sum()
    assert float((n - R * w).abs().max()) <= 1.5  # a token's interval holds its share of the grid, give or take one
