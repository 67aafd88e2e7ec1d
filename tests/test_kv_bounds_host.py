"""The bounds of kv_tight: attention as the kernel rounds it is within them, and each planted mistake is not."""
import pytest
import torch

import kv_tight as T
from test_gpu_kv_attention import make

LENGTHS = [2, 17, 40, 600, 5000]


def simulate(x, weights=lambda p: p, values=lambda v: v):
    """The rows' attention with weights and values changed on the way: [rows, heads, D], rounded as the result is."""
    H, S, D = x["k"].shape[1:]
    G, c, n = x["q"].shape[1] // H, x["context"][0], len(x["q"])
    ids = x["table"][0, :-(-c // S)].long()
    out = torch.zeros(x["q"].shape, dtype=torch.float64)
    for h in range(H):
        k, v = (y[ids, h].double().reshape(-1, D)[:c] for y in (x["k"], x["v"]))
        if x["k_scale"] is not None:
            k, v = k * x["k_scale"].double()[h], v * x["v_scale"].double()[h]
        for j in range(n):
            p = c - n + j + 1
            z = x["q"][j, h * G:(h + 1) * G].double() @ k[:p].T * D ** -0.5
            w = torch.exp(z - z.amax(1, keepdim=True)).float()
            out[j, h * G:(h + 1) * G] = weights(w).double() @ values(v[:p].clone()) / w.double().sum(1, keepdim=True)
    return out.to(x["q"].dtype).double()


def one(w):
    return w.bfloat16().float()


def two(w):
    return one(w) + one(w - one(w))


def within(x, got):
    out, e = T.attend(x)
    return bool(((got - out).abs() <= e).all())


def inputs(kind, c, dtype, D=64):
    return getattr(T, kind)(make([c], [1], H=2, G=2, D=D, dtype=dtype, seed=c, junk=False))


@pytest.mark.parametrize("kind", ["marked", "cancelling", "alternating"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "fp32"])
def test_right_results_are_within(kind, dtype):
    for c in LENGTHS:
        x = inputs(kind, c, dtype)
        assert within(x, simulate(x, two if dtype != "fp32" else lambda w: w)), c


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_weights_of_eight_bits_are_not(dtype):
    for c in LENGTHS:
        for kind in ("cancelling", "alternating")[c > 1000:]:  # many roundings of either sign are nearly none
            x = inputs(kind, c, dtype)
            assert not within(x, simulate(x, one)), (c, kind)


def swapped(a, b):
    def f(v):
        v[[a, b]] = v[[b, a]]
        return v
    return f


def dropped(*at):
    def f(v):
        v[list(at)] = 0
        return v
    return f


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "fp32"])
@pytest.mark.parametrize("c", LENGTHS[1:])
def test_values_in_the_wrong_place_are_not(c, dtype):
    x = inputs("marked", c, dtype)
    for at in (0, c // 2, c - 1):
        assert not within(x, simulate(x, values=dropped(at))), at
    for a, b in ((0, 1), (c // 2, c // 2 + 4), (c - 17, c - 1), (3, c - 2)):
        assert not within(x, simulate(x, values=swapped(a, b))), (a, b)
    half = lambda v: torch.cat([v[:, 32:], v[:, :32]], 1)  # noqa: E731
    pairs = lambda v: v.view(len(v), -1, 2).flip(2).reshape(len(v), -1)  # noqa: E731
    assert not within(x, simulate(x, values=half)) and not within(x, simulate(x, values=pairs))
