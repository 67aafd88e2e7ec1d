"""dsde_kv_attention over values that are not finite: what a row sees of them in a dimension is its output there
(inf, -inf, NaN with both or a NaN), wherever they lie and whatever their weights; everything else is unchanged, bit for bit."""
import math

import pytest
import torch

from test_gpu_kv_attention import DT, make, to_gpu

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def put(x, places):
    """A copy of the inputs with the values ``places``: (token of the only sequence, key head, dimension, value)."""
    x = dict(x, v=x["v"].clone())
    S = x["v"].shape[2]
    for t, h, d, value in places:
        x["v"][int(x["table"][0, t // S]), h, t % S, d] = value
    return x


def expected(x, places, window):
    """What each output (row, head, dimension) has to be; 0 where no such value is seen."""
    T, heads, D = x["q"].shape
    H, c = x["v"].shape[1], x["context"][0]
    plus, minus = torch.zeros(T, heads, D, dtype=torch.bool), torch.zeros(T, heads, D, dtype=torch.bool)
    last = {place[:3]: place[3] for place in places}  # a place has one value, the last one put there
    for j in range(T):
        p = c - T + j
        for (t, h, d), value in last.items():
            if t <= p and (not window or t > p - window):
                at = slice(h * (heads // H), (h + 1) * (heads // H))
                plus[j, at, d] |= value != -INF
                minus[j, at, d] |= value != INF
    want = torch.zeros(T, heads, D)
    want[plus], want[minus], want[plus & minus] = INF, -INF, NAN
    return want


def check(lib, x, places, scale=None, window=0):
    print(x["q"].shape, x["k"].shape, x["context"], places, window, flush=True)
    clean = lib.kv_attention(**to_gpu(x), scale=scale, window=window, lse=True)
    got = lib.kv_attention(**to_gpu(put(x, places)), scale=scale, window=window, lse=True)
    want, o = expected(x, places, window), got["out"].float().cpu()
    odd = want != 0
    assert bool((~torch.isfinite(want[odd])).all()) and bool(odd.any())
    wrong = odd & ~((o == want) | (torch.isnan(o) & torch.isnan(want)))
    assert not bool(wrong.any()), [(i, float(o[tuple(i)]), float(want[tuple(i)])) for i in wrong.nonzero().tolist()[:5]]
    assert torch.equal(o[~odd], clean["out"].float().cpu()[~odd])
    assert torch.equal(got["lse"], clean["lse"]) and not got["seq_err"].any()


SHAPES = [(40, 1, 1, 1, 64), (40, 9, 2, 2, 64), (130, 3, 2, 2, 16), (500, 1, 2, 1, 80), (700, 1, 2, 4, 128), (700, 9, 1, 4, 128),
          (600, 6, 1, 8, 128), (700, 9, 1, 8, 128), (600, 8, 1, 8, 64), (400, 5, 2, 8, 64), (900, 1, 1, 8, 256), (900, 4, 1, 8, 256), (3000, 1, 1, 8, 128),
          (3000, 9, 2, 4, 128), (2500, 64, 1, 1, 64), (9000, 2, 1, 2, 192)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("c,n,H,G,D", SHAPES)
def test_infinities_anywhere(gpu_lib, c, n, H, G, D, dtype):
    """In the first, middle and last tiles, of one sign and of both, in items of one wavefront and of many."""
    x = make([c], [n], H=H, G=G, D=D, dtype=dtype, seed=c + n, junk=False)
    h, mid = H - 1, c // 2
    places = [(0, h, 0, INF), (mid, h, 1, -INF), (0, h, 2, INF), (mid, h, 2, -INF), (c // 3, h, 3, NAN), (c - 1, h, 4, INF),
              (5, h, D - 1, -INF), (5, h, 7, INF), (c // 3, h, 7, INF), (c - 1, h, 7, INF), (c - 1, h, 8, INF), (1, h, 8, -INF),
              (mid + 1, h, 9, NAN), (mid + 1, h, 10, INF)]
    check(gpu_lib, x, places)
    for place in ((0, 0, 5, INF), (mid, 0, 6, -INF), (c - 1, 0, 11, INF)):  # alone in a call
        check(gpu_lib, x, [place])


@pytest.mark.parametrize("D", [16, 64, 128, 256])
@pytest.mark.parametrize("c,n,G", [(40, 1, 1), (700, 9, 8), (3000, 2, 2)])
def test_nan_of_eight_bits_anywhere(gpu_lib, c, n, G, D):
    x = make([c], [n], H=2, G=G, D=D, dtype="e4m3", seed=c, junk=False)
    check(gpu_lib, x, [(0, 1, 0, NAN), (c // 2, 1, 3, NAN), (c - 1, 1, D - 1, NAN), (c // 3, 0, 5, NAN)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [1, 16, 33, 100])
def test_infinities_and_a_window(gpu_lib, window, dtype):
    for c, n, G in ((150, 4, 2), (600, 9, 8), (2000, 20, 1)):
        x = make([c], [n], H=1, G=G, D=64, dtype=dtype, seed=c, junk=False)
        t = c - window - n // 2  # seen by the first rows alone
        places = [(max(0, t), 0, 1, INF), (c - 1, 0, 2, -INF), (c - 1 - window // 2, 0, 2, INF), (c - n, 0, 3, INF), (0, 0, 4, NAN)]
        check(gpu_lib, x, places, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("slope", [-4.0, -0.3, 0.3, 4.0])
@pytest.mark.parametrize("c", [60, 900, 5000])
def test_weights_that_vanish(gpu_lib, c, slope, dtype):
    """Scores that rise or fall by hundreds: weights and factors that underflow to 0 beside an infinity, in one
    wavefront and between parts."""
    x = make([c], [2], H=1, G=2, D=64, dtype=dtype, junk=False)
    x["q"].zero_()
    x["q"][:, :, 0] = 1.0
    ids = x["table"][0, :-(-c // 16)].long()
    k = x["k"].float()
    k[ids, 0, :, 0] = (torch.arange(len(ids) * 16).view(-1, 16) * slope)
    x["k"] = k.to(DT[dtype])
    check(gpu_lib, x, [(0, 0, 1, INF), (c - 3, 0, 2, -INF), (c // 2, 0, 3, INF), (3, 0, 4, INF), (c - 5, 0, 4, -INF)], scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [40, 700, 3000])
def test_scores_that_are_not_finite_beside_them(gpu_lib, c, dtype):
    """A key of -inf (weight 0) whose value is inf: seen all the same.  A NaN score: its row is NaN throughout."""
    x = make([c], [2], H=1, G=1, D=64, dtype=dtype, junk=False)
    x["q"][:, 0, 3] = 1.0
    x["k"][int(x["table"][0, 0]), 0, 4, 3] = -INF
    check(gpu_lib, x, [(4, 0, 5, INF), (c // 2, 0, 6, INF)])
    y = to_gpu(put(x, [(4, 0, 5, INF), (c // 2, 0, 6, -INF)]))
    y["q"][1, 0, 9] = NAN
    got = gpu_lib.kv_attention(**y, lse=True)
    assert float(got["out"][0, 0, 5]) == INF and float(got["out"][0, 0, 6]) == -INF and bool(torch.isfinite(got["out"][0, 0, 7:]).all())
    assert bool(torch.isnan(got["out"][1]).all()) and bool(torch.isnan(got["lse"][1]).all()) and bool(torch.isfinite(got["lse"][0]).all())


def test_many_sequences_each_with_its_own(gpu_lib):
    """An infinity in every third sequence: the others keep their bits, however shares are cut."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(1, 700, (120,), generator=g).tolist()
    x = make(lens, [1 + i % 3 for i in range(120)], H=2, G=2, D=128, seed=3, junk=False)
    clean = gpu_lib.kv_attention(**to_gpu(x), lse=True)
    for b in range(0, 120, 3):
        x["v"][int(x["table"][b, 0]), 1, 0, b] = INF if b % 2 else -INF
    got = gpu_lib.kv_attention(**to_gpu(x), lse=True)
    o, want = got["out"].float().cpu(), clean["out"].float().cpu()
    for b in range(0, 120, 3):
        c, n = lens[b], 1 + b % 3
        for j in range(n):
            if c - n + j >= 0:
                want[x["cu"][b] + j, 2:, b] = INF if b % 2 else -INF
    assert torch.equal(o, want) and torch.equal(got["lse"], clean["lse"])


@pytest.mark.parametrize("c", [40, 700, 5000])
def test_a_scale_past_the_types_range(gpu_lib, c):
    """Values that pass the largest number once they are scaled are infinite with their sign, in one wavefront and in parts."""
    x = make([c], [1], H=1, G=2, D=64, dtype="e4m3", junk=False)
    x["v"] = torch.where(torch.arange(64) % 2 == 0, 256.0, -256.0).expand(x["v"].shape).to(DT["e4m3"])
    x["v_scale"] = torch.full((1,), 2.0 ** 121)  # 2^129
    o = gpu_lib.kv_attention(**to_gpu(x))["out"].float().cpu()
    assert bool((o[..., 0::2] == INF).all()) and bool((o[..., 1::2] == -INF).all())
