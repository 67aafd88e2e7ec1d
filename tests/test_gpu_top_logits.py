"""dsde_top_logits against its definition in 64 bits."""
import math

import pytest
import torch

from rows_reference import top_row

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def check(lib, z, k, T=1.0, rows=None, **kw):
    o = lib.top_logits(z.cuda() if z.device.type == "cpu" else z, k, temperature=T, **kw)
    torch.cuda.synchronize()
    o = {n: v.cpu() for n, v in o.items()}
    for i in range(len(z)) if rows is None else rows:
        v, ids, lse = top_row(z[i].cpu().float(), k, T)
        assert int(o["row_err"][i]) == 0
        assert torch.equal(o["values"][i].double(), v) and torch.equal(o["ids"][i].long(), ids), i
        # fp32 rounding of the result, and a few 1e-7 of the sum
        assert abs(float(o["lse"][i]) - float(lse)) <= 1e-7 * abs(float(lse)) + 1e-6, i
    return o


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,k", [(1, 1), (2, 1), (7, 7), (8, 3), (9, 9), (65, 64), (256, 256), (300, 256), (1000, 1),
                                 (8191, 100), (8193, 256), (32000, 8), (50257, 33), (128256, 64), (70001, 256)])
def test_the_largest_logits(gpu_lib, V, k, dtype):
    g = torch.Generator().manual_seed(V + k)
    z = (3.0 * torch.randn(5, V, generator=g)).to(DT[dtype])
    check(gpu_lib, z, k, T=(1.0, 2.0, 0.5)[V % 3])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_k_beyond_the_row(gpu_lib, dtype):
    z = torch.randn(3, 20, generator=torch.Generator().manual_seed(0)).to(DT[dtype])
    o = check(gpu_lib, z, 33)
    assert (o["ids"][:, 20:] == -1).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [100, 5000, 40000])
def test_ties_and_masks(gpu_lib, V, dtype):
    """Constant rows, rows of few values, clustered maxima, masks that leave less than k tokens."""
    g = torch.Generator().manual_seed(V)
    z = torch.randn(8, V, generator=g)
    z[0] = 0.0
    z[0, ::3] = -0.0
    z[1] = -3.3895313892515355e38
    z[2] = torch.randint(0, 3, (V,), generator=g).float()
    z[3, V // 2:] = -math.inf
    z[4] = -math.inf
    z[4, V - 5:] = torch.tensor([1.0, 3.0, 2.0, 3.0, -1.0])
    z[5] = torch.arange(V).float() / V  # the largest next to each other
    z[6, :V // 2] = -3.3895313892515355e38
    z[7] = -z[5] - 2.0
    check(gpu_lib, z.to(DT[dtype]), 64)
    check(gpu_lib, z.to(DT[dtype]), 1)


def test_nearby_fp32_keys(gpu_lib):
    """Thousands of fp32 logits that share the upper half of their keys."""
    g = torch.Generator().manual_seed(9)
    z = 1.0 + torch.rand(4, 20000, generator=g) * 2e-3
    z[1] = -z[1]
    z[2, 100:15000] = 1.0
    z[3] = (z[3] * 65536).round() / 65536
    check(gpu_lib, z, 256)


def test_data_errors_flag_their_row_alone(gpu_lib):
    z = torch.randn(4, 9000, generator=torch.Generator().manual_seed(1))
    z[0, 0] = math.nan
    z[1, 8999] = math.inf
    z[2] = -math.inf
    o = gpu_lib.top_logits(z.cuda(), 5)
    assert o["row_err"].tolist() == [gpu_lib.ERR_LOGIT] * 3 + [0]
    assert (o["ids"][:3] == -1).all() and o["values"][:3].isnan().all() and o["lse"][:3].isnan().all()
    v, ids, _ = top_row(z[3], 5, 1.0)
    assert torch.equal(o["ids"][3].cpu().long(), ids)


def test_strided_rows_and_streams(gpu_lib):
    g = torch.Generator().manual_seed(8)
    wide = torch.randn(6, 9031, generator=g).to(torch.bfloat16).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for kw in ({}, dict(stream=side)):
        check(gpu_lib, wide[:, 5:9006], 40, **kw)
    assert gpu_lib.top_logits(wide[:0], 4)["ids"].shape == (0, 4)


def test_offsets_beyond_32_bits(gpu_lib):
    """More than 2^31 logits and 2^32 bytes, in several passes of the workspace."""
    R, V = 34000, 65536
    z = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(3)
    rows = [0, 11000, 12000, 32768, 33999]
    for i in rows:
        z[i] = torch.randn(V, generator=g).to(torch.bfloat16).cuda()
    check(gpu_lib, z, 16, rows=rows)
