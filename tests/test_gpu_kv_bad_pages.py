"""Pages that are none, in every form of the attention kernel: the rows that see one are NaN, every other keeps its bits."""
import pytest
import torch

from test_gpu_kv_attention import make, to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("n,G", [(5, 1), (4, 6), (20, 2), (8, 8), (9, 8)])
def test_rows_that_see_it_alone(gpu_lib, n, G, D, dtype):
    """The page of the newest tokens of a sequence, one seen by all, one outside of a window; other sequences around it."""
    c = 32 * 16 + n // 2  # the newest page begins at token 512, behind some of the rows
    x = make([70, c, 33], [1, n, 2], H=2, G=G, D=D, dtype=dtype, seed=n * G, junk=False)
    y = to_gpu(x)
    want = gpu_lib.kv_attention(**y, lse=True)
    first, last = x["cu"][1], x["cu"][2]
    for at, id_ in ((32, -1), (32, x["k"].shape[0]), (3, 2 ** 31 - 1)):
        z = dict(y, table=y["table"].clone())
        z["table"][1, at] = id_
        got = gpu_lib.kv_attention(**z, lse=True)
        assert got["seq_err"].tolist() == [0, 256, 0]
        sees = torch.tensor([first <= t < last and c - n + (t - first) >= 16 * at for t in range(len(x["q"]))], device="cuda")
        assert 0 < int(sees.sum()) <= n
        for k in ("out", "lse"):
            assert bool(torch.isnan(got[k][sees]).all()) and torch.equal(got[k][~sees], want[k][~sees]), (at, k)
    seen = gpu_lib.kv_attention(**y, lse=True, window=40)
    got = gpu_lib.kv_attention(**z, lse=True, window=40)  # page 3 is outside
    assert not got["seq_err"].any() and torch.equal(got["out"], seen["out"]) and torch.equal(got["lse"], seen["lse"])
