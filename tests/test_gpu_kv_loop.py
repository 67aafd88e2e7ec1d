"""The cache's calls as a serving loop makes them: map, write, attention, verification, and the next step from its counts."""
import contextlib

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
B, H, G, D, V, S, K_MAX, WIDTH = 6, 2, 3, 64, 400, 16, 6, 9
ROWS = B * (K_MAX + 1)
PROMPTS = [0, 1, 15, 16, 40, 33]
P = 40
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -8}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
I32 = dict(dtype=torch.int32, device="cuda")


class Model:
    """One attention layer over a token's and a position's random rows; the draft is a table of token pairs."""

    def __init__(self, dtype):
        g = torch.Generator().manual_seed(5)
        self.dtype = DT[dtype]
        self.row = torch.float32 if dtype == "fp32" else torch.bfloat16
        n = (H * G + 2 * H) * D
        self.token = torch.randn(V, n, generator=g).cuda()
        self.position = torch.randn(S * WIDTH, n, generator=g).cuda()
        self.head = (0.5 * torch.randn(H * G * D, V, generator=g)).cuda()
        self.pairs = (2 * torch.randn(V, V, generator=g)).cuda()
        self.scales = [torch.tensor([0.5, 0.25], device="cuda") if dtype == "e4m3" else None for _ in range(2)]

    def rows(self, tokens, positions):
        x = (self.token[tokens] + self.position[positions.clamp(min=0).long()]).to(self.row).view(-1, H * G + 2 * H, D)
        return x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]  # three views of one array

    def stored(self, x):
        """What the cache holds of rows [n, H, D] (the scales are powers of two)."""
        if self.dtype is not torch.float8_e4m3fn:
            return x.cpu()
        return (x.float() / self.scales[0][:, None]).clamp(-448, 448).cpu().to(self.dtype)


class Step:
    """A step's device work, for as many rows as it may have, on buffers that stay."""

    def __init__(self, lib, model, window):
        self.lib, self.m, self.window = lib, model, window
        self.pool = lib.new_kv_pool(B, WIDTH, P)
        self.cache = lib.new_kv_cache(P, S, H, D, model.dtype)
        for c in self.cache:
            c.view(torch.uint8).fill_(0xff)  # NaN until written
        self.kv_len, self.accepted, self.sl = torch.zeros(B, **I32), torch.full((B,), -1, **I32), torch.zeros(B, **I32)
        self.tokens = torch.zeros(ROWS, dtype=torch.int64, device="cuda")
        self.map = dict(lib.new_kv_map_out(B, ROWS), base=self.kv_len)
        self.map_ws = lib.new_kv_map_workspace(B)
        self.ws = lib.new_kv_attention_workspace(B, H, G, K_MAX + 1, D)
        self.row_err = torch.zeros(ROWS, **I32)
        self.out = {"out": torch.zeros(ROWS, H * G, D, dtype=model.row, device="cuda"), "seq_err": torch.zeros(B, **I32),
                    "lse": torch.zeros(ROWS, H * G, device="cuda")}

    def prompt(self, lengths, tokens):
        """Prompts into the cache: one call of each, with room of their own."""
        out = self.lib.kv_map(torch.tensor(lengths, **I32), self.kv_len, self.pool, S, sum(lengths), extra=0)
        _, k, v = self.m.rows(tokens, out["positions"])
        err = self.lib.kv_write(k, v, out["slots"], *self.cache, *self.m.scales)
        assert not out["seq_err"].any() and not err.any()
        self.kv_len.copy_(out["context"])
        return k, v

    def forward(self):
        self.lib.kv_map(self.sl, self.kv_len, self.pool, S, ROWS, accepted=self.accepted, out=self.map, workspace=self.map_ws)
        self.q, self.k, self.v = self.m.rows(self.tokens, self.map["positions"])
        self.lib.kv_write(self.k, self.v, self.map["slots"], *self.cache, *self.m.scales, row_err=self.row_err)
        self.lib.kv_attention(self.q, *self.cache, self.pool["table"], self.map["context"], self.map["cu_rows"], K_MAX + 1,
                              window=self.window, k_scale=self.m.scales[0], v_scale=self.m.scales[1], out=self.out, workspace=self.ws)


def loop(lib, dtype, window, mode, steps=9):
    """The loop's tokens and outputs; each step is checked against the histories that the host keeps."""
    model = Model(dtype)
    step = Step(lib, model, window)
    g = torch.Generator().manual_seed(11)
    prompt = torch.randint(0, V, (sum(PROMPTS),), generator=g).cuda()
    k, v = step.prompt(PROMPTS, prompt)
    cu = R.prefix(PROMPTS)
    history = [(model.stored(k)[a:b], model.stored(v)[a:b]) for a, b in zip(cu, cu[1:])]
    last = torch.randint(0, V, (B,), generator=g).tolist()
    ring = [torch.zeros(B, 32, device="cuda"), torch.zeros(B, **I32), torch.zeros(B, **I32)]
    sl, log = [3, 0, 6, 1, 2, 6], []
    stream = torch.cuda.Stream() if mode == "stream" else None
    graph = None
    if mode == "graph":
        # a first run of the libraries, on state that is put back
        kept = {n: t.clone() for n, t in step.pool.items()}, step.kv_len.clone()
        step.forward()
        torch.cuda.synchronize()
        for n, t in kept[0].items():
            step.pool[n].copy_(t)
        step.kv_len.copy_(kept[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.forward()
    for i in range(steps):
        # the draft: a chain of tokens for each sequence
        rows, drafts, q_rows = [], [], []
        for b in range(B):
            t = last[b]
            rows.append(t)
            for _ in range(sl[b]):
                q_rows.append(t)
                t = int(torch.multinomial(torch.softmax(model.pairs[t].cpu(), 0), 1, generator=g))
                drafts.append(t)
                rows.append(t)
        n = len(rows)
        step.sl.copy_(torch.tensor(sl, **I32))
        step.tokens.zero_()
        step.tokens[:n] = torch.tensor(rows, device="cuda")
        for t in step.out.values():
            t.fill_(7)
        if graph is not None:
            graph.replay()
        else:
            torch.cuda.synchronize()
            with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
                step.forward()
        torch.cuda.synchronize()
        # pages and rows
        cu, base = R.prefix([x + 1 for x in sl]), [len(x[0]) for x in history]
        context = [x + y + 1 for x, y in zip(base, sl)]
        held = [-(-c // S) for c in context]
        assert step.map["base"].tolist() == base and step.map["context"].tolist() == context
        assert step.map["cu_rows"].tolist() == cu and not step.map["seq_err"].any() and not step.row_err.any()
        assert step.pool["held"].tolist() == held and int(step.pool["n_free"]) == P - sum(held)
        ids = [step.pool["table"][b, :held[b]].tolist() for b in range(B)]
        assert sorted(sum(ids, []) + step.pool["free"][:P - sum(held)].tolist()) == list(range(P))
        # attention, over the histories and the new rows
        history = [tuple(torch.cat([x, model.stored(y[cu[b]:cu[b + 1]])]) for x, y in zip(history[b], (step.k, step.v)))
                   for b in range(B)]
        most = max(context)
        dense = [torch.stack([torch.nn.functional.pad(x[j].float(), (0, 0, 0, 0, 0, most - len(x[j]))).transpose(0, 1) for x in history])
                 for j in range(2)]
        scales = [None if s is None else s.cpu() for s in model.scales]
        out, lse, e_out, e_lse = R.attend(step.q[:n].cpu(), *dense, torch.arange(B)[:, None], context, cu, D ** -0.5, window, *scales,
                                          EPS[dtype])
        got = step.out["out"].cpu().double(), step.out["lse"].cpu().double()
        assert bool(((got[0][:n] - out).abs() <= e_out).all()) and bool(((got[1][:n] - lse).abs() <= e_lse).all())
        assert bool((got[0][n:] == 7).all()) and bool((got[1][n:] == 7).all()) and not step.out["seq_err"].any()
        # verification, and what the next step takes from it
        pairs = model.pairs[step.tokens[:n]]
        target = step.out["out"][:n].float().view(n, -1) @ model.head + pairs
        draft = model.pairs[torch.tensor(q_rows, dtype=torch.int64, device="cuda")].contiguous()
        u = torch.rand(2, max(len(drafts), B), generator=g).cuda()
        r = lib.step(target, draft, step.sl, torch.tensor(R.prefix(sl), **I32), torch.tensor(drafts, **I32), torch.ones(B, device="cuda"),
                     u[0, :len(drafts)].contiguous(), u[1, :B].contiguous(), K_MAX, *ring, torch.full((B,), float(K_MAX), device="cuda"),
                     sl_min=1.0)
        assert not r["seq_err"].any()
        accepted = r["accepted"].tolist()
        step.accepted.copy_(r["accepted"])
        last = [int(r["tokens"][b, accepted[b]]) for b in range(B)]
        history = [tuple(x[:base[b] + accepted[b] + 1] for x in history[b]) for b in range(B)]
        log.append((step.out["out"][:n].clone(), step.out["lse"][:n].clone(), list(last), accepted))
        # now and then a sequence drafts nothing, or as much as it may: its pages come and go
        sl = [0 if (i + b) % 5 == 0 else K_MAX if (i + b) % 5 == 3 else x for b, x in enumerate(r["sl_next"].tolist())]
    taken = sum((x[3] for x in log), [])
    assert 0 < sum(taken) and min(taken) == 0  # both outcomes occur
    return log


def same(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and x[2:] == y[2:]


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("window", [0, 20])
def test_serving_loop(gpu_lib, dtype, window):
    loop(gpu_lib, dtype, window, "eager")


def test_captured_and_on_another_stream(gpu_lib):
    """A step captured once and replayed for rows and pages that differ each time, and one on another stream: the eager
    loop's bits."""
    eager = loop(gpu_lib, "bf16", 0, "eager")
    same(eager, loop(gpu_lib, "bf16", 0, "stream"))
    same(eager, loop(gpu_lib, "bf16", 0, "graph"))
