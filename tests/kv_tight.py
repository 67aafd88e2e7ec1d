"""Bounds of the cache attention's outputs that tell its roundings apart, and inputs on which a wrong one shows.

A weight of a 16-bit cache is the sum of two bf16 numbers: of x in [2^e, 2^(e+1)) the first leaves 2^(e-8) at most, of which the
second leaves 2^(e-17) at most, so the weight is good to 2^-17 of itself (fp32: to 2^-24).  That error counts against
A = sum p |v|; the result's own rounding, half a step of its type, counts against |out| alone."""
import torch

import kv_reference as R

WEIGHT = {"bf16": 2.0 ** -17, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -17}
RESULT = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -8}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


def attend(x, scale=None, window=0):
    """out and the bound of its error, of inputs as test_gpu_kv_attention.make gives them."""
    D = x["q"].shape[2]
    out, _, e, _ = R.attend(x["q"], x["k"], x["v"], x["table"], x["context"], x["cu"], D ** -0.5 if scale is None else scale, window,
                            x["k_scale"], x["v_scale"], WEIGHT[x["dtype"]])
    # weights under 2^-100 of the largest may be lost altogether; values here are under 2^10
    return out, e * (1 + RESULT[x["dtype"]]) + RESULT[x["dtype"]] * out.abs() + 2.0 ** -90


def _tokens(x, name):
    """Every token's place (page, position) in order, for each sequence."""
    S = x[name].shape[2]
    for b, c in enumerate(x["context"]):
        t = torch.arange(c)
        yield b, x["table"][b][t // S].long(), t % S


def marked(x):
    """Values that are 0 but in one dimension, another for each neighbour: out says what weight each token's value got."""
    v = torch.zeros(x["v"].shape)
    D = v.shape[3]
    for b, page, at in _tokens(x, "v"):
        t = torch.arange(len(page))
        for h in range(v.shape[1]):
            v[page, h, at, (5 * t + 3 + h + b) % D] = (1 + (7 * t + h) % 5).float()
    return dict(x, v=v.to(DT[x["dtype"]]), q=(0.3 * x["q"].float()).to(x["q"].dtype))


def cancelling(x):
    """Neighbours with values that differ in sign alone and weights that differ by a few percent: out is far smaller than
    sum p |v|, so that the weights' rounding is not covered by the result's."""
    k, v = x["k"].float().clone(), x["v"].float().clone()
    for _, page, at in _tokens(x, "k"):
        n = len(page) // 2 * 2
        a, b = (page[0:n:2], at[0:n:2]), (page[1:n:2], at[1:n:2])
        k[b[0], :, b[1]] = k[a[0], :, a[1]]
        k[b[0], :, b[1], 1] += 0.5
        v[b[0], :, b[1]] = -v[a[0], :, a[1]]
    return dict(x, k=k.to(DT[x["dtype"]]), v=v.to(DT[x["dtype"]]), q=(0.3 * x["q"].float()).to(x["q"].dtype))


def alternating(x):
    """One key but for a step in every second token, and values whose sign alternates: roundings of the same weights add
    up over any length."""
    k, v = x["k"].float().clone(), x["v"].float().clone()
    for _, page, at in _tokens(x, "k"):
        k[page, :, at] = k[page[:1], :, at[:1]]
        k[page[1::2], :, at[1::2], 1] += 0.5
        v[page, :, at] = v[page, :, at].abs()
        v[page[1::2], :, at[1::2]] *= -1
    return dict(x, k=k.to(DT[x["dtype"]]), v=v.to(DT[x["dtype"]]), q=(0.3 * x["q"].float()).to(x["q"].dtype))
