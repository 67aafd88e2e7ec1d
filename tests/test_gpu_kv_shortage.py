"""A step for which a sequence finds no pages, and the steps behind it: its tokens stay what was written of them."""
import random

import pytest
import torch

import kv_reference as R
from test_gpu_kv_map import I32, state, to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("aliased", [False, True])
@pytest.mark.parametrize("B,room", [(5, 0), (130, 0), (130, 10_000), (1500, 0), (1500, 10_000)])
def test_counts_of_flagged_sequences_are_not_added(gpu_lib, B, room, aliased):
    """Steps with too few pages, in which flagged sequences come back with counts that mean nothing; pages become free as
    sequences end.  Against the loop that adds nothing for them."""
    r = random.Random(B)
    W, page = 9, 16
    P = B * W
    lens, pool = state(r, B, W, page, P, 80, spare=2)
    kept = pool["n_free"][0]
    gpu = to_gpu(pool)
    kv_len, accepted = torch.tensor(lens, **I32), [-1] * B
    out = flagged = None
    ever = set()
    for step in range(6):
        sl = [r.randrange(0, 40) for _ in range(B)]
        ending = [b for b in range(B) if step >= 2 and r.random() < 0.05]
        if ending:  # their pages go back first: no tokens, no rows
            zero = [0 if b in ending else n for b, n in enumerate(lens)]
            acc = [-1 if b in ending else a for b, a in enumerate(accepted)]
            new = gpu_lib.kv_map(torch.full((B,), 0, **I32), torch.tensor(zero, **I32), gpu, page, 0, extra=0,
                                 accepted=torch.tensor(acc, **I32), last_err=None if out is None else out["seq_err"])
            pool, want = R.kv_map([0] * B, 0, zero, [-1 if flagged and flagged[b] else a for b, a in enumerate(acc)], pool["table"],
                                  pool["held"], pool["free"], pool["n_free"][0], page, P, 0)
            assert new["base"].tolist() == want["base"] and new["seq_err"].tolist() == want["seq_err"]
            lens, accepted, flagged = want["base"], [-1] * B, None
            kv_len, out = torch.tensor(lens, **I32), None
        rows = sum(sl) + B + room
        last = None if out is None else out["seq_err"]
        o = gpu_lib.new_kv_map_out(B, rows)
        if aliased:
            o["base"] = kv_len
            if last is not None:
                o["seq_err"] = last
        out = gpu_lib.kv_map(torch.tensor(sl, **I32), kv_len, gpu, page, rows, accepted=torch.tensor(accepted, **I32), last_err=last, out=o)
        torch.cuda.synchronize()
        pool, want = R.kv_map(sl, 1, lens, [-1 if flagged and flagged[b] else a for b, a in enumerate(accepted)], pool["table"],
                              pool["held"], pool["free"], pool["n_free"][0], page, P, rows)
        for k, v in want.items():
            assert out[k].tolist() == v, (step, k)
        for k, v in pool.items():
            assert gpu[k].tolist() == v, (step, k)
        flagged, lens, kv_len = want["seq_err"], want["base"], out["base"]
        ever |= {b for b in range(B) if flagged[b]}
        # what a step makes of a flagged sequence's rows: anything
        accepted = [r.randrange(-5, 24) if flagged[b] else r.randrange(0, s + 1) for b, s in enumerate(sl)]
    assert kept < P and ever


def test_a_shortage_ends_and_nothing_unwritten_is_seen(gpu_lib):
    """Map, write and attention over a cache of NaN: every token that a row sees was written, step by step."""
    B, W, page, P, H, D, room = 3, 8, 16, 7, 1, 16, 3 * 20
    pool = gpu_lib.new_kv_pool(B, W, P)
    kc, vc = gpu_lib.new_kv_cache(P, page, H, D)
    kc.fill_(float("nan"))
    vc.fill_(float("nan"))
    kv_len, out = torch.zeros(B, **I32), dict(gpu_lib.new_kv_map_out(B, room))
    out["base"] = kv_len
    out["seq_err"].zero_()
    accepted = torch.full((B,), -1, **I32)
    sls = [[15, 15, 15], [17, 17, 17], [2, -1, 17], [1, 0, 4], [3, 2, 1]]
    lens, seen = [0, 0, 0], []
    for step, sl in enumerate(sls):
        if step == 2:
            kv_len[1], accepted[1] = 0, -1  # the second sequence ends (and draws a new request, without rows yet)
            lens[1] = 0
        gpu_lib.kv_map(torch.tensor(sl, **I32), kv_len, pool, page, room, accepted=accepted, last_err=out["seq_err"], out=out)
        x = out["positions"].clamp(min=0).bfloat16()[:, None, None].expand(room, H, D).contiguous()
        assert not gpu_lib.kv_write(x, x, out["slots"], kc, vc).any()
        got = gpu_lib.kv_attention(torch.zeros(room, H, D, dtype=torch.bfloat16, device="cuda"), kc, vc, pool["table"], out["context"],
                                   out["cu_rows"], 20)
        err, cu = out["seq_err"].tolist(), out["cu_rows"].tolist()
        assert out["base"].tolist() == lens
        assert not got["seq_err"].any()
        seen.append(err)
        for b in range(B):
            for j in range(sl[b] + 1):
                o = got["out"][cu[b] + j, 0].float().cpu()
                p = lens[b] + j  # equal weights: the mean position, exact up to the result's rounding and the sum's
                want = 0.0 if err[b] else p / 2
                assert bool(((o - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want).all()), (step, b, j)
        # every flagged sequence accepts what it may
        accepted.copy_(torch.tensor([s for s in sl], **I32))
        lens = [n if e else n + s + 1 for n, s, e in zip(lens, sl, err)]
    assert seen[1] == [0, 0, 256] and not any(sum(seen[2:], []))


def test_a_captured_map_remembers_whom_it_flagged(gpu_lib):
    """One graph that reads the flags it wrote in the replay before, with eager work between replays, through shortages."""
    r = random.Random(21)
    B, W, page, room = 70, 9, 16, 70 * 41
    P = B * W
    lens, pool = state(r, B, W, page, P, 80, spare=2)
    gpu = to_gpu(pool)
    keep = {k: v.clone() for k, v in gpu.items()}
    sl, acc, kv_len = (torch.zeros(B, **I32) for _ in range(3))
    out, ws = gpu_lib.new_kv_map_out(B, room), gpu_lib.new_kv_map_workspace(B)
    out["base"] = kv_len

    def step():
        gpu_lib.kv_map(sl, kv_len, gpu, page, room, accepted=acc, last_err=out["seq_err"], out=out, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, v in keep.items():
        gpu[k].copy_(v)
    out["seq_err"].zero_()
    kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    accepted, flagged, ever, again = [-1] * B, [0] * B, 0, 0
    for i in range(6):
        drafts = [r.randrange(0, 40) for _ in range(B)]
        sl.copy_(torch.tensor(drafts, dtype=torch.int32))
        acc.copy_(torch.tensor(accepted, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        pool, want = R.kv_map(drafts, 1, lens, [-1 if f else a for f, a in zip(flagged, accepted)], pool["table"], pool["held"], pool["free"],
                              pool["n_free"][0], page, P, room)
        for k, v in want.items():
            assert out[k].tolist() == v, (i, k)
        for k, v in pool.items():
            assert gpu[k].tolist() == v, (i, k)
        again += sum(bool(a) and not b for a, b in zip(flagged, want["seq_err"]))
        lens, flagged = want["base"], want["seq_err"]
        ever += sum(map(bool, flagged))
        accepted = [r.randrange(-9, 40) if f else r.randrange(0, d + 1) for f, d in zip(flagged, drafts)]
    assert ever and again


def test_flags_that_are_refused(gpu_lib):
    sl, n = torch.ones(3, **I32), torch.zeros(3, **I32)
    for bad, text in ((torch.zeros(3, dtype=torch.int64, device="cuda"), "last_err must be torch.int32, got torch.int64"),
                      (torch.zeros(2, **I32), "last_err has 2 elements, needs 3"), (torch.zeros(3, dtype=torch.int32), "must be a GPU tensor"),
                      (torch.zeros(6, **I32)[::2], "last_err must be contiguous")):
        with pytest.raises(gpu_lib.DsdeError, match=text):
            gpu_lib.kv_map(sl, n, gpu_lib.new_kv_pool(3, 4, 12), 16, 6, last_err=bad)
    out = gpu_lib.kv_map(sl, n, gpu_lib.new_kv_pool(3, 4, 12), 16, 6, last_err=torch.zeros(3, dtype=torch.uint32, device="cuda"))
    assert not out["seq_err"].any() and out["base"].tolist() == [0, 0, 0]
