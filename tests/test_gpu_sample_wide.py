"""dsde_sample where the filters keep many tokens: cuts beyond the sorted candidates."""
import pytest
import torch

from rows_reference import check_draw

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (temperature, top_k, top_p, min_p)
WIDE = [(2.0, 0, 0.9, 1e-4), (3.0, 0, 0.999, 1e-3), (1.5, 0, 0.3, 1e-5), (1.0, 5000, 1.0, 1e-3), (8.0, 20000, 0.5, 0.0),
        (1.0, 257, 1.0, 0.0), (5.0, 0, 0.999999, 0.0), (50.0, 0, 0.5, 0.0), (50.0, 700, 0.99, 0.02), (6.0, 0, 1.0, 1e-6),
        (2.0, 9000, 0.9, 1e-3), (0.01, 6000, 1.0, 0.0)]


def check(lib, z, par, seed):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(len(par), generator=g)
    T, k, p, m = (torch.tensor(x, dtype=d) for x, d in zip(zip(*par), (torch.float32, torch.int32, torch.float32, torch.float32)))
    o = lib.sample(z.cuda(), T.cuda(), u.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=m.cuda(), kept=True)
    again = lib.sample(z.cuda(), T.cuda(), u.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=m.cuda())
    torch.cuda.synchronize()
    assert torch.equal(o["tokens"], again["tokens"]) and torch.equal(o["logprob"], again["logprob"])
    for i in range(len(par)):
        assert int(o["row_err"][i]) == 0
        check_draw(z[i].float(), float(T[i]), int(k[i]), float(p[i]), float(m[i]), float(u[i]), int(o["tokens"][i]),
                   float(o["logprob"][i]), int(o["kept"][i]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [700, 6001, 20011, 50257, 131072, 170003])
def test_many_kept_tokens(gpu_lib, V, dtype):
    g = torch.Generator().manual_seed(V)
    z = (3.0 * torch.randn(len(WIDE), V, generator=g)).to(DT[dtype])
    check(gpu_lib, z, WIDE, V)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_kept_tokens_of_few_values(gpu_lib, dtype):
    """Rows of a handful of values, nearly flat rows and rows sorted by id: long runs of ties at the cuts."""
    g = torch.Generator().manual_seed(1)
    V = 60000
    few = torch.randint(0, 5, (len(WIDE), V), generator=g).float()
    flat = 0.01 * torch.randn(len(WIDE), V, generator=g)
    falling = (-torch.arange(V).float() / 3000).expand(len(WIDE), V)
    for seed, z in enumerate((few, flat, falling.contiguous(), falling.flip(1).contiguous())):
        check(gpu_lib, z.to(DT[dtype]), WIDE, seed)


@pytest.mark.parametrize("V", [1200000, 3000001])
def test_many_kept_tokens_of_a_wide_vocabulary(gpu_lib, V):
    g = torch.Generator().manual_seed(V)
    par = WIDE[:4] + WIDE[7:9]
    check(gpu_lib, (2.0 * torch.randn(len(par), V, generator=g)).to(torch.bfloat16), par, V)
