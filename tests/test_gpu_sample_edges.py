"""dsde_sample and dsde_top_logits at the ends of their ranges: rows whose largest logit holds nearly all mass,
uniforms of 0 on rows whose weights underflow, filters below the histogram's range."""
import math

import pytest
import torch

from rows_reference import check_draw, sample_row

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def arrays(par):
    """The settings (temperature, top_k, top_p, min_p) of every row, on the GPU."""
    types = (torch.float32, torch.int32, torch.float32, torch.float32)
    return [torch.tensor(x, dtype=d, device="cuda") for x, d in zip(zip(*par), types)]


def draw(lib, z, par, u):
    T, k, p, m = arrays(par)
    o = lib.sample(z.cuda(), T, torch.as_tensor(u, dtype=torch.float32).cuda(), top_k=k, top_p=p, min_p=m, kept=True)
    assert (o["row_err"] == 0).all()
    return {k: v.cpu() for k, v in o.items()}


def check(o, z, par, u):
    for i, row in enumerate(par):
        T, k, p, m = (float(torch.tensor(x, dtype=torch.float32)) for x in row)
        check_draw(z[i].float(), T, int(k), p, m, float(torch.tensor(u[i], dtype=torch.float32)), int(o["tokens"][i]),
                   float(o["logprob"][i]), int(o["kept"][i]))


# log p = -log1p(rest), and the row's lse = log1p(rest) where its largest logit is 0: as exact as the sum of the other
# weights.  A weight e^-x is off by (1.5 x + 1) 2^-23 of itself (as WEIGHT_TOL, which is this at x = 17), the nine rounds
# of fp32 additions over a segment of 512 by 9 2^-24, the result's rounding by 2^-24.
def rest_tol(x):
    return (1.5 * x + 1) * 2.0 ** -23 + 10 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("par", [(1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 40, 1.0, 0.0), (0.7, 0, 0.9, 0.0),
                                 (1.0, 0, 1.0, 0.05), (1.0, 700, 1.0, 0.0), (1.0, 3000, 0.99, 0.0)])
def test_logprob_of_a_token_that_holds_nearly_all_mass(gpu_lib, par, dtype):
    V, gaps = 70001, (14.0, 16.0, 18.0, 20.0, 22.0, 24.0, 30.0, 38.0)
    g = torch.Generator().manual_seed(5)
    z = torch.randn(len(gaps), V, generator=g) - torch.tensor(gaps)[:, None]
    at = torch.randint(0, V, (len(gaps),), generator=g)
    z = z.scatter(1, at[:, None], 0.0).to(DT[dtype])
    o = draw(gpu_lib, z, [par] * len(gaps), [0.5] * len(gaps))
    T = par[0] or 1.0
    rest = (z.double() / float(torch.tensor(T))).exp().scatter(1, at[:, None], 0.0).sum(1)
    assert torch.equal(o["tokens"].long(), at)
    want = torch.log1p(rest)
    tol = rest_tol(torch.tensor(gaps).double() / T) * want
    assert bool(((o["logprob"].double() + want).abs() <= tol).all()), o["logprob"].double() / want + 1
    if par == (1.0, 0, 1.0, 0.0):
        lse = gpu_lib.top_logits(z.cuda(), 8)["lse"].cpu().double()
        assert bool(((lse - want).abs() <= tol).all()), lse / want - 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logprob_of_several_equal_maxima(gpu_lib, dtype):
    """n equal maxima in one group, one segment, one chunk and several: log p = -log n - log1p(rest / n)."""
    V = 30011
    places = ([5], [8, 9, 15], [600, 700, 1000], [0, 8191, 8192, 30010], list(range(512, 1024)), list(range(9000, 21000)))
    z = torch.randn(len(places), V, generator=torch.Generator().manual_seed(6)) - 22.0
    for row, p in zip(z, places):
        row[p] = 0.0
    z = z.to(DT[dtype])
    n = torch.tensor([len(p) for p in places], dtype=torch.float64)
    for par in ((1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0)):
        o = draw(gpu_lib, z, [par] * len(places), [0.5] * len(places))
        assert all(int(t) in p for t, p in zip(o["tokens"], places))
        rest = z.double().exp().sum(1) - n
        want = n.log() + torch.log1p(rest / n)
        assert bool(((o["logprob"].double() + want).abs() <= rest_tol(22.0) * want).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [0.05, 0.01, 2.0 ** -10])
@pytest.mark.parametrize("masked", [0, 1, 600, 9000])
def test_uniform_of_zero_where_weights_underflow(gpu_lib, masked, T, dtype):
    """Segments whose weight is the product of two tiny numbers hold no token of positive weight: the draw passes them
    over.  The first tokens are masked, so that none of them may be drawn."""
    V, R = 128256, 24
    g = torch.Generator().manual_seed(masked + 1)
    z = 4.0 * torch.randn(R, V, generator=g)
    z[:, :masked] = -math.inf
    z = z.to(DT[dtype])
    for par in ((T, 0, 1.0, 0.0), (T, 50, 1.0, 0.0), (T, 3000, 1.0, 0.0)):
        o = draw(gpu_lib, z, [par] * R, [0.0] * R)
        check(o, z, [par] * R, [0.0] * R)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [6001, 50257, 131072])
def test_min_p_below_the_histogram(gpu_lib, V, dtype):
    """min_p under 2^-32 with a top_k whose last token lies more than 32 octaves below the maximum: top_k cuts where it
    is the shorter one, and min_p where that is."""
    par = [(0.2, 300, 1.0, 1e-12), (0.1, 300, 1.0, 1e-30), (0.1, 2000, 1.0, 1e-20), (0.1, 600, 1.0, 1e-25),
           (0.05, 1000, 1.0, 1e-37), (0.2, 1200, 1.0, 2.0 ** -31), (0.2, 1200, 1.0, 2.0 ** -32), (0.1, 300, 1.0, 1e-12),
           (0.1, 700, 0.999999, 1e-30), (0.1, 0, 0.999999, 1e-30), (0.1, 0, 1.0, 1e-30)]
    g = torch.Generator().manual_seed(V)
    z = (3.0 * torch.randn(len(par), V, generator=g)).to(DT[dtype])
    u = torch.rand(len(par), generator=g).tolist()
    cut = [sample_row(z[i].float(), T, k, p, float(torch.tensor(m)))[3] for i, (T, k, p, m) in enumerate(par)]
    assert 300 in cut or V < 10000  # top_k is what cuts at least one of the wider ones
    check(draw(gpu_lib, z, par, u), z, par, u)
