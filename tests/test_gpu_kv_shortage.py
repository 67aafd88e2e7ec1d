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
