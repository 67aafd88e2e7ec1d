"""The operators around a verification step whose speed is followed: drawing tokens from
a model's logits, keeping a row's largest logits, and distilling a draft model from them.

A case is a dict of plain values:

  op       sample   dsde.sample: one token per row, under per-row temperature, top-k,
                    top-p and min-p, from given uniforms
           top      dsde.top_logits: the k largest logits of each row and its log-normaliser
           loss     dsde.distill_loss: the divergence from a teacher's top logits
           train    dsde.distill with its backward, through autograd
           step     dsde.distill_step: loss and gradient in one call
  R, V     rows, vocabulary
  dtype    bf16 or fp32 logits (gradients have the same type)
  padded   the rows are V wide slices of rows whose width is a multiple of 64
  filters  (sample) how the rows are drawn, see _filters
  K        (top, loss, train, step) entries kept per row
  tail     (loss, train, step) whether the teacher's log-normaliser is given
  T        (loss, train, step) temperature
  pads     (step) every pads-th row has weight 0 (padding of a packed batch); 0: none

Logits are Gaussian with a Zipf rank bias per row; a student's are its teacher's
with noise of a strength of its own per row.
"""
import math
import random

import torch

own = False

ROWS = 256  # rows made or checked at once
FILTERS = ("none", "nucleus", "topk", "minp", "mixed", "broad", "greedy")


def _case(name, op, R, V, dtype="bf16", padded=False, filters="", K=0, tail=False, T=1.0, pads=0):
    c = dict(op=op, R=R, V=V, dtype=dtype, padded=padded, filters=filters, K=K, tail=tail, T=T, pads=pads)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's request: the draft model's next token, nothing but latency
        _case("sample_one", "sample", 1, 128256, filters="nucleus"),
        # a mid-sized batch whose sampler upcasts its logits, rows of an odd width cut from padded ones
        _case("sample_b64_fp32", "sample", 64, 50257, "fp32", padded=True, filters="mixed"),
        # a few sequences at a high temperature: nuclei of thousands of tokens
        _case("sample_broad", "sample", 32, 128256, filters="broad"),
        # the 256-sequence batch, each request with settings of its own
        _case("sample_b256", "sample", 256, 128256, filters="mixed"),
        # one drafting step of the controller loop's 1,024 sequences: the drafts that a
        # verification accepts or rejects are drawn from the whole distribution
        _case("sample_b1024", "sample", 1024, 128256, filters="none"),
        # every target row of the 256-sequence step, kept for training
        _case("top_b256", "top", 1408, 128256, K=64),
        # a teacher that hands out fp32 logits, many entries
        _case("top_fp32", "top", 320, 152064, "fp32", K=256),
        # a validation pass over the drafted positions of that step
        _case("loss_b256", "loss", 1152, 128256, K=64, tail=True),
        # training a small draft model in fp32 through autograd
        _case("train_fp32", "train", 32, 32000, "fp32", K=16, T=2.0),
        # training through autograd on the drafted positions of one step
        _case("train_b256", "train", 1152, 128256, K=64, tail=True),
        # a packed batch with padding between its sequences, odd sizes throughout
        _case("step_odd", "step", 333, 50257, padded=True, K=33, T=1.5, pads=7),
        # the most rows: one micro-batch of a training run
        _case("step_4096", "step", 4096, 128256, K=64, tail=True),
    ]


MOST_BYTES = 4096 * 128256 * 4


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "loss", "train", "step"])
    most = 1024 if op == "sample" else 4096
    R = round(math.exp(rng.uniform(0, math.log(most))))
    V = round(math.exp(rng.uniform(math.log(8192), math.log(152064))))
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if rng.random() < 0.6:
        V -= V % 64
    per = (2 if dtype == "bf16" else 4) * (2 if op in ("train", "step") else 1)
    while R * V * per > (MOST_BYTES if op in ("train", "step") else MOST_BYTES // 4):
        R = (R + 1) // 2
    padded = op != "train" and rng.random() < 0.2
    K = rng.choice([1, 4, 8, 16, 33, 64, 64, 100, 128, 256])
    if op == "sample":
        return _case(None, op, R, V, dtype, padded, filters=rng.choice(FILTERS))
    if op == "top":
        return _case(None, op, R, V, dtype, padded, K=K)
    return _case(None, op, R, V, dtype, padded, "", K, rng.random() < 0.5, rng.choice([1.0, 1.0, 1.5, 2.0]),
                 rng.choice([0, 0, 5, 7]) if op == "step" and R >= 16 else 0)


def _filters(case, seed):
    """Temperature, top_k, top_p and min_p of every row."""
    one = {
        "none": [(1.0, 0, 1.0, 0.0)],  # the whole distribution
        "nucleus": [(0.7, 0, 0.9, 0.0)],  # the usual chat settings
        "topk": [(0.8, 50, 1.0, 0.0), (1.0, 20, 1.0, 0.0), (1.0, 500, 1.0, 0.0)],
        "minp": [(1.0, 0, 1.0, 0.05), (1.2, 0, 1.0, 0.02)],
        # requests of many users in one batch
        "mixed": [(0.7, 0, 0.9, 0.0), (1.0, 40, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.8, 200, 0.95, 0.0),
                  (1.0, 0, 1.0, 0.05), (1.0, 0, 0.95, 0.0)],
        "broad": [(1.2, 0, 0.95, 0.0), (1.3, 0, 0.98, 0.0), (1.0, 0, 0.99, 0.0), (1.5, 4000, 0.97, 0.0)],
        "greedy": [(0.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0)],
    }[case["filters"]]
    first = random.Random(seed).randrange(len(one))
    return [one[(first + i) % len(one)] for i in range(case["R"])]


def _rows(case, g, r, seed_rows, dtype, dev):
    """Empty logits of the case's layout, and a maker of the fp32 values of rows i..j."""
    V = case["V"]
    wide = -(-V // 64) * 64 if case["padded"] else V
    buf = torch.empty((seed_rows, wide), dtype=dtype, device=dev)
    if wide > V:
        buf[:, V:] = 0.0
    steps = [r.randrange(1, V) for _ in range(seed_rows)]
    steps = torch.tensor([a if math.gcd(a, V) == 1 else 1 for a in steps], device=dev)[:, None]
    shift = torch.randint(0, V, (seed_rows, 1), generator=g, device=dev)
    ids = torch.arange(V, device=dev)[None, :]

    def values(i, j):
        rank = (steps[i:j] * ids + shift[i:j]) % V + 1
        z = torch.randn((j - i, V), generator=g, device=dev)
        return z.mul_(4.0).sub_(rank.float().log_(), alpha=1.05)

    return buf[:, :V], values


def _token(z, T, k, p, m, u):
    """The token that every row's uniform stands for, in 64 bits.  T 0 counts as 1."""
    V = z.shape[1]
    x = z.double()
    x = (x - x.amax(1, keepdim=True)) / torch.where(T > 0, T, 1.0).double()[:, None]
    _, order = torch.sort(z, dim=1, descending=True, stable=True)
    e = x.exp().gather(1, order)
    c = e.cumsum(1)
    at = torch.where((k > 0) & (k < V), k.long(), V) - 1
    last = torch.searchsorted(c, (p.double() * c.gather(1, at[:, None])[:, 0])[:, None])[:, 0]
    last = torch.minimum(at, torch.where(p < 1, last, V - 1))
    last = torch.minimum(last, torch.where(m > 0, (e >= m.double()[:, None]).sum(1), V) - 1).clamp_(min=0)
    e.masked_fill_(torch.arange(V, device=z.device)[None, :] > last[:, None], 0.0)
    c = torch.zeros_like(e).scatter_(1, order, e).cumsum_(1)
    return torch.searchsorted(c, (u.double() * c[:, -1])[:, None], right=True)[:, 0].clamp_(max=V - 1)


def _uniforms(case, z, par, g):
    """A uniform for every row.  Where another one or another top_p within 5e-6 would
    give another token, the outcome is a matter of rounding: such are drawn again."""
    R = z.shape[0]
    u = torch.empty(R, device=z.device)
    for i in range(0, R, ROWS):
        rows, (T, k, p, m) = z[i:i + ROWS], (x[i:i + ROWS] for x in par)
        v = torch.rand(rows.shape[0], generator=g, device=z.device)
        todo = torch.arange(rows.shape[0], device=z.device)
        for _ in range(20):
            if not len(todo):
                break
            a = (rows[todo], T[todo], k[todo])
            sure = torch.ones(len(todo), dtype=torch.bool, device=z.device)
            first = None
            for dp in (-5e-6, 5e-6):
                pp = torch.where(p[todo] < 1, p[todo].double() * (1 + dp), 1.0)
                for du in (-5e-6, 5e-6):
                    t = _token(*a, pp, m[todo], (v[todo].double() + du).clamp(0, 1 - 1e-9))
                    first = t if first is None else first
                    sure &= t == first
            todo = todo[~sure]
            v[todo] = torch.rand(len(todo), generator=g, device=z.device)
        u[i:i + ROWS] = v
    return u


def _inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(1_000_003 * seed + 29)
    r = random.Random(seed)
    R, V, K = case["R"], case["V"], case["K"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    z, values = _rows(case, g, r, R, dt, dev)
    if case["op"] in ("sample", "top"):
        for i in range(0, R, ROWS):
            z[i:i + ROWS] = values(i, min(i + ROWS, R))
        if case["op"] == "top":
            return dict(logits=z)
        par = list(zip(*_filters(case, seed)))
        par = [torch.tensor(x, dtype=d, device=dev) for x, d in zip(par, (torch.float32, torch.int32, torch.float32, torch.float32))]
        return dict(logits=z, temperature=par[0], top_k=par[1], top_p=par[2], min_p=par[3],
                    u=_uniforms(case, z, par, g))
    ids = torch.empty((R, K), dtype=torch.int32, device=dev)
    teacher = torch.empty((R, K), device=dev)
    lse = torch.empty(R, device=dev)
    sigma = 0.2 + 1.8 * torch.rand((R, 1), generator=g, device=dev)
    for i in range(0, R, ROWS):
        j = min(i + ROWS, R)
        t = values(i, j)
        z[i:j] = t + sigma[i:j] * torch.randn((j - i, V), generator=g, device=dev)
        t = t.to(dt).float()
        teacher[i:j], top = torch.topk(t, K, dim=1)
        ids[i:j] = top.int()
        lse[i:j] = torch.logsumexp(t.double() / case["T"], dim=1)
    live = torch.arange(R, device=dev) % case["pads"] != 0 if case["pads"] else torch.ones(R, dtype=torch.bool, device=dev)
    weight = live.float() / live.sum().clamp(min=1)
    return dict(logits=z, ids=ids, teacher=teacher, lse=lse if case["tail"] else None, weight=weight, T=case["T"])


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"], K=case["K"])
    if case["op"] == "train":
        s["logits"].requires_grad_(True)
    return s


def _sample(s):
    z, T = s["logits"].float(), s["temperature"]
    V = z.shape[1]
    top = z.amax(1, keepdim=True)
    e = ((z - top) / torch.where(T > 0, T, 1.0)[:, None]).exp_()
    total = e.sum(1)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices  # equal logits: lowest id first
    w = e.gather(1, order)
    # cumulative weights in 64 bits: which token a uniform meets should not depend on how a long sum is rounded
    c = w.cumsum(1, dtype=torch.float64)
    n = torch.arange(V, device=z.device)[None, :]
    k = torch.where((s["top_k"] > 0) & (s["top_k"] < V), s["top_k"], V)[:, None]
    kept = n < k
    p = s["top_p"][:, None]
    kept &= (p >= 1) | (c - w < p * c.gather(1, k.long() - 1))
    kept &= w >= s["min_p"][:, None]
    kept |= n == 0
    c = torch.zeros_like(w).scatter_(1, order, w * kept).cumsum(1, dtype=torch.float64)
    token = (c <= s["u"][:, None] * c[:, -1:]).sum(1)
    token = torch.where(T > 0, token, order[:, 0])[:, None]
    return dict(tokens=token[:, 0].int(), logprob=e.gather(1, token)[:, 0].log() - total.log())


def _top(s):
    z = s["logits"].float()
    values, ids = torch.sort(z, dim=1, descending=True, stable=True)
    top = values[:, :1]
    return dict(values=values[:, :s["K"]].contiguous(), ids=ids[:, :s["K"]].int(),
                lse=(z - top).exp_().sum(1).log() + top[:, 0])


def _distill(s, weight):
    """Loss of every row and, with weights, the gradient of their weighted sum."""
    x = s["logits"].detach().float() / s["T"]
    ids, t = s["ids"].long(), s["teacher"] / s["T"]
    top = x.amax(1, keepdim=True)
    q = (x - top).exp_()
    at = x.gather(1, ids) - top
    total = q.sum(1, keepdim=True)
    rest = q.scatter(1, ids, 0.0).sum(1, keepdim=True)
    if s["lse"] is None:
        t = t - t.amax(1, keepdim=True)
        logp = t - t.exp().sum(1, keepdim=True).log()
        p = logp.exp()
        loss = (p * (logp - at + total.log())).sum(1)
        share = torch.ones_like(total)
    else:
        logp = t - s["lse"][:, None]
        p = logp.exp()
        r = (1.0 - p.sum(1, keepdim=True)).clamp_(min=0.0)
        tail = torch.where(r > 0, r * (r.clamp(min=1e-30).log() - rest.log() + total.log()), 0.0)
        loss = (p * (logp - at + total.log())).sum(1) + tail[:, 0]
        share = 1.0 - r * total / rest
    if weight is None:
        return loss
    scale = (weight / s["T"])[:, None]
    grad = q.mul_(scale * share / total)
    grad.scatter_(1, ids, scale * (at.exp() / total - p))
    return loss, grad.to(s["logits"].dtype)


def _plain(s):
    if s["op"] == "sample":
        return _sample(s)
    if s["op"] == "top":
        return _top(s)
    if s["op"] == "loss":
        return dict(loss=_distill(s, None))
    loss, grad = _distill(s, s["weight"])
    if s["op"] == "step":  # rows of weight 0 are left out
        loss = torch.where(s["weight"] != 0, loss, 0.0)
    return dict(loss=loss, grad=grad)


def run(s):
    if not own:
        return _plain(s)
    import paper_2509_01083_amd as dsde
    z = s["logits"]
    if s["op"] == "sample":
        o = dsde.sample(z, s["temperature"], s["u"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return dict(tokens=o["tokens"], logprob=o["logprob"])
    if s["op"] == "top":
        o = dsde.top_logits(z, s["K"])
        return dict(values=o["values"], ids=o["ids"], lse=o["lse"])
    if s["op"] == "loss":
        o = dsde.distill_loss(z, s["ids"], s["teacher"], teacher_lse=s["lse"], temperature=s["T"])
        return dict(loss=o["loss"])
    if s["op"] == "train":
        z.grad = None
        loss = dsde.distill(z, s["ids"], s["teacher"], teacher_lse=s["lse"], temperature=s["T"])
        loss.backward(s["weight"])
        return dict(loss=loss.detach(), grad=z.grad)
    o = dsde.distill_step(z, s["ids"], s["teacher"], s["weight"], teacher_lse=s["lse"], temperature=s["T"])
    return dict(loss=o["loss"], grad=o["grad"])


def work(case):
    """Each row once, the small arrays, and for training the gradient's rows once; an
    exponential, a product and two sums per logit, twice where there is a gradient."""
    R, V, K = case["R"], case["V"], case["K"]
    live = R - -(-R // case["pads"]) if case["pads"] else R
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        return {"bytes": R * V * e + 32 * R, "flops": 4 * R * V}
    if case["op"] == "top":
        return {"bytes": R * V * e + 8 * R * K + 4 * R, "flops": 4 * R * V}
    n = {"loss": 1, "train": 3, "step": 2}[case["op"]]  # autograd's backward reads the logits again
    grad = R if case["op"] in ("train", "step") else 0
    return {"bytes": live * V * e * (n - 1 if grad else 1) + grad * V * e + 8 * R * K + 12 * R,
            "flops": (8 if grad else 4) * live * V}


def exact(case, seed):
    x = _inputs(case, seed)
    z, R, V = x["logits"], case["R"], case["V"]
    dev = z.device
    out = []
    for i in range(0, R, ROWS):
        rows = z[i:i + ROWS]
        y = {k: v[i:i + ROWS] if isinstance(v, torch.Tensor) else v for k, v in x.items()}
        if case["op"] == "sample":
            T = y["temperature"].double()
            best = rows.double().eq(rows.double().amax(1, keepdim=True)).int().argmax(1)
            t = torch.where(T > 0, _token(rows, y["temperature"], y["top_k"], y["top_p"], y["min_p"], y["u"]), best)
            lp = torch.log_softmax(rows.double() / torch.where(T > 0, T, 1.0)[:, None], dim=1)
            out.append(dict(tokens=t.int(), logprob=lp.gather(1, t[:, None])[:, 0]))
            continue
        if case["op"] == "top":
            v, order = torch.sort(rows.double(), dim=1, descending=True, stable=True)
            out.append(dict(values=v[:, :case["K"]], ids=order[:, :case["K"]].int(), lse=torch.logsumexp(v, dim=1)))
            continue
        T, ids = case["T"], y["ids"].long()
        logq = torch.log_softmax(rows.double() / T, dim=1)
        t = y["teacher"].double() / T
        inside = torch.zeros_like(logq, dtype=torch.bool).scatter_(1, ids, True)
        logp = torch.log_softmax(t, dim=1) if y["lse"] is None else t - y["lse"].double()[:, None]
        p = logp.exp()
        loss = (p * (logp - logq.gather(1, ids))).sum(1)
        grad = logq.exp()
        if y["lse"] is not None:
            r = (1 - p.sum(1)).clamp(min=0)
            logr = torch.logsumexp(logq.masked_fill(inside, -math.inf), dim=1)
            loss = loss + torch.where(r > 0, r * (r.clamp(min=1e-300).log() - logr), 0.0)
            grad = torch.where(inside, grad, grad * (1 - r / logr.exp())[:, None])
        if case["op"] == "loss":
            out.append(dict(loss=loss))
            continue
        grad.scatter_add_(1, ids, -p)
        live = y["weight"] != 0 if case["op"] == "step" else torch.ones(len(rows), dtype=torch.bool, device=dev)
        out.append(dict(loss=torch.where(live, loss, 0.0), grad=grad.mul_((y["weight"].double() / T)[:, None])))
    return {k: torch.cat([o[k] for o in out]) for k in out[0]}
