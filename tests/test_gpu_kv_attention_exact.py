"""dsde_kv_attention within bounds that count each rounding where it occurs, on inputs on which a weight of too few bits
or a value in the wrong place shows (tests/test_kv_bounds_host.py plants both)."""
import pytest
import torch

import kv_tight as T
from test_gpu_kv_attention import make, to_gpu

pytestmark = pytest.mark.gpu
TYPES = ["bf16", "fp32", "e4m3"]
KINDS = ["marked", "cancelling", "alternating"]


def check(lib, x, window=0):
    print(x["q"].shape, x["k"].shape, x["context"], window, flush=True)
    got = lib.kv_attention(**to_gpu(x), window=window)
    out, e = T.attend(x, window=window)
    d = (got["out"].cpu().double() - out).abs()
    assert bool((d <= e).all()), (float((d / e).max()), (d > e).nonzero()[:5].tolist())
    assert not got["seq_err"].any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128, 160, 192, 240, 256])
def test_head_sizes(gpu_lib, D, dtype, kind):
    x = make([2, 17, 40, 333], [1, 1, 2, 3], H=2, G=3, D=D, dtype=dtype, seed=D, junk=False, by_token=D % 32 == 0)
    check(gpu_lib, getattr(T, kind)(x))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 16), (3, 8), (5, 8), (8, 8), (9, 8), (33, 1)])
def test_row_counts(gpu_lib, n, G, D, dtype, kind):
    """1 to 72 rows of a key head: every number of row blocks."""
    check(gpu_lib, getattr(T, kind)(make([150, 77], [n, max(1, n // 2)], H=1, G=G, D=D, S=32, dtype=dtype, seed=n * G, junk=False)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c,D", [(600, 64), (5000, 64), (5000, 128), (1500, 256)])
def test_long_caches(gpu_lib, c, D, dtype, kind):
    check(gpu_lib, getattr(T, kind)(make([c], [2], H=2, G=2, D=D, S=64, dtype=dtype, seed=c, junk=False)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [2, 33, 200])
def test_windows(gpu_lib, window, dtype, kind):
    check(gpu_lib, getattr(T, kind)(make([400, 90], [5, 3], H=1, G=2, D=64, dtype=dtype, seed=window, junk=False)), window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_near_the_stated_limit(gpu_lib, dtype):
    """Sizes that add up to just under 2^120: finite, and as exact as any."""
    x = make([200, 30], [3, 1], H=1, G=2, D=64, dtype=dtype, seed=1, junk=False)
    x["v"] = (x["v"].float().sign() * 2.0 ** 112).to(x["v"].dtype)  # 200 of them: 2^119.7
    got = gpu_lib.kv_attention(**to_gpu(x))["out"].cpu().double() * 2.0 ** -112
    x["v"] = x["v"].float().sign().to(x["v"].dtype)
    out, e = T.attend(x)
    assert bool(((got - out).abs() <= e).all())
