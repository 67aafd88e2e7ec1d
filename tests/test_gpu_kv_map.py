"""dsde_kv_map against a loop over the sequences."""
import random

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def state(r, B, W, page, P, most, spare=None):
    """A pool in use: random lengths, pages from a shuffled cache."""
    lens = [r.randrange(0, most + 1) for _ in range(B)]
    held = [min(W, -(-n // page) + r.randrange(0, 3)) for n in lens]
    ids = list(range(P))
    r.shuffle(ids)
    table = []
    for h in held:
        table.append(ids[:h] + [-1] * (W - h))
        ids = ids[h:]
    assert len(ids) >= 0 and all(len(t) == W for t in table)
    if spare is not None:
        ids = ids[:spare]
    return lens, dict(table=table, held=held, free=ids + [-7] * (P - len(ids)), n_free=[len(ids)])


def to_gpu(pool):
    return {k: torch.tensor(v, **I32) for k, v in pool.items()}


def check(lib, pool, sl, extra, kv_len, accepted, page, P, rows, gpu=None, **kw):
    """One call on the GPU and in the loop; the loop's pool, and the GPU's."""
    gpu = to_gpu(pool) if gpu is None else gpu
    acc = None if accepted is None else torch.tensor(accepted, **I32)
    got = lib.kv_map(torch.tensor(sl, **I32), torch.tensor(kv_len, **I32), gpu, page, rows, extra=extra, accepted=acc, **kw)
    torch.cuda.synchronize()
    new, want = R.kv_map(sl, extra, kv_len, [-1] * len(sl) if accepted is None else accepted, pool["table"], pool["held"],
                         pool["free"], pool["n_free"][0], page, P, rows)
    for k, v in want.items():
        if k in got:
            assert got[k].tolist() == v, k
        else:
            assert rows == 0 and k in ("slots", "positions")
    for k, v in new.items():
        assert gpu[k].tolist() == v, k
    return new, gpu, got


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 256, 1023, 1024, 1025, 2500])
def test_steps_follow_the_loop(gpu_lib, B, page):
    r = random.Random(B * page)
    W, most = 6, 4 * page
    P = B * W
    lens, pool = state(r, B, W, page, P, most)
    accepted, gpu = [-1] * B, None
    for step in range(4):
        sl = [r.randrange(0, 9) for _ in range(B)]
        rows = sum(sl) + B + r.randrange(0, 20)
        pool, gpu, got = check(gpu_lib, pool, sl, 1, lens, accepted, page, P, rows, gpu)
        lens = got["base"].tolist()
        accepted = [r.randrange(-1, s + 1) for s in sl]


@pytest.mark.parametrize("B,most", [(3, 9000), (40, 1500), (1, 60000), (1100, 70), (300, 1500), (1100, 400)])
def test_prompts_and_their_end(gpu_lib, B, most):
    """More rows than the planning workgroup maps itself; then every page goes back, by that workgroup or by all."""
    r = random.Random(B)
    page = 16
    W = -(-most // page)
    P = B * W + 5
    pool = dict(table=[[-1] * W for _ in range(B)], held=[0] * B, free=list(range(P))[::-1], n_free=[P])
    sl = [r.randrange(most // 2, most + 1) for _ in range(B)]
    start = {k: [list(x) for x in v] if k == "table" else list(v) for k, v in pool.items()}
    pool, gpu, _ = check(gpu_lib, pool, sl, 0, [0] * B, None, page, P, sum(sl))
    pool, gpu, _ = check(gpu_lib, pool, [0] * B, 0, [0] * B, None, page, P, 0, gpu)
    assert pool == start  # as it was


def test_a_call_that_gives_back_undoes_the_one_before(gpu_lib):
    r = random.Random(5)
    B, W, page = 300, 8, 16
    lens, pool = state(r, B, W, page, B * W, 100)
    held = [-(-n // page) for n in lens]  # nothing beyond what the tokens need
    for b in range(B):
        for c in range(held[b], pool["held"][b]):
            pool["free"][pool["n_free"][0]] = pool["table"][b][c]
            pool["n_free"][0] += 1
            pool["table"][b][c] = -1
    pool["held"] = held
    first = to_gpu(pool)
    sl = [r.randrange(0, 17) for _ in range(B)]
    new, gpu, _ = check(gpu_lib, pool, sl, 1, lens, None, page, B * W, sum(sl) + B)
    assert new != pool
    check(gpu_lib, new, [0] * B, 0, lens, None, page, B * W, 0, gpu)
    n = pool["n_free"][0]
    for k in first:
        assert torch.equal(first[k][:n] if k == "free" else first[k], gpu[k][:n] if k == "free" else gpu[k]), k


@pytest.mark.parametrize("spare", [0, 1, 7, 40])
def test_pages_run_out(gpu_lib, spare):
    r = random.Random(spare)
    B, W, page = 130, 9, 16
    lens, pool = state(r, B, W, page, B * W, 80, spare)
    sl = [r.randrange(0, 40) for _ in range(B)]
    _, _, got = check(gpu_lib, pool, sl, 1, lens, None, page, B * W, sum(sl) + B)
    assert (got["seq_err"] == 256).any() and (got["seq_err"] == 0).any()


@pytest.mark.parametrize("change", [dict(n_free=[-1]), dict(n_free=[10 ** 6]), dict(n_free=[540]), dict(held=[-1, 10]),
                                    dict(lens=[-1, -5]), dict(accepted=[-2, -9]), dict(sl=[-2, -100]), dict(sl=[500, 2 ** 31 - 2]),
                                    dict(rows=37), dict(rows=0), dict(sl=[2 ** 31 - 1] * 60), dict(lens=[2 ** 31 - 1] * 3)])
def test_faults_are_flagged(gpu_lib, change):
    """Values out of range, at the first sequences: nothing outside the arrays is touched, others go on."""
    r = random.Random(3)
    B, W, page = 60, 9, 16
    lens, pool = state(r, B, W, page, B * W, 100)
    sl, accepted, rows = [r.randrange(0, 9) for _ in range(B)], [-1] * B, 1000
    for k, v in change.items():
        if k in pool:
            pool[k] = v + pool[k][len(v):]
        elif k == "lens":
            lens = v + lens[len(v):]
        elif k == "accepted":
            accepted = v + accepted[len(v):]
        elif k == "sl":
            sl = v + sl[len(v):]
        else:
            rows = v
    P = B * W
    gpu = to_gpu(pool)
    got = gpu_lib.kv_map(torch.tensor(sl, **I32), torch.tensor(lens, **I32), gpu, page, rows,
                         accepted=torch.tensor(accepted, **I32))
    torch.cuda.synchronize()
    new, want = R.kv_map(sl, 1, lens, accepted, pool["table"], pool["held"], pool["free"], pool["n_free"][0], page, P, rows)
    want["cu_rows"] = [min(x, 2 ** 31 - 1) for x in want["cu_rows"]]
    want["base"] = [min(x, 2 ** 31 - 1) for x in want["base"]]
    for k, v in want.items():
        if k in got:
            assert got[k].tolist() == v, k
    for k, v in new.items():
        assert gpu[k].tolist() == v, k
    assert any(want["seq_err"])


def test_page_ids_out_of_range(gpu_lib):
    """A table and a stack that hold what is no page: rows there get no slot."""
    B, W, page, P = 3, 4, 16, 12
    pool = dict(table=[[0, 99, -1, -1], [1, -1, -1, -1], [3, 4, -1, -1]], held=[2, 1, 2],
                free=[5, 12, -3] + [-7] * 9, n_free=[3])
    _, _, got = check(gpu_lib, pool, [3, 3, 3], 1, [30, 14, 30], None, page, P, 12)
    assert got["seq_err"].tolist() == [256, 256, 0]  # the third takes page 5


@pytest.mark.parametrize("B", [130, 1500])
@pytest.mark.parametrize("fault", ["spare 0", "spare 60", "n_free", "held", "ids", "sl"])
def test_faults_with_much_room(gpu_lib, B, fault):
    """The same outcomes where the whole card maps the rows."""
    r = random.Random(B)
    W, page = 9, 16
    P = B * W
    lens, pool = state(r, B, W, page, P, 80, int(fault[6:]) if fault.startswith("spare") else None)
    sl = [r.randrange(0, 40) for _ in range(B)]
    if fault == "n_free":
        pool["n_free"] = [P + 1]
    elif fault == "held":
        pool["held"][:2], pool["held"][-1] = [-1, W + 1], 2 ** 31 - 1
    elif fault == "ids":
        for b in range(0, B, 3):
            pool["table"][b] = [x if x < 0 or r.random() < 0.5 else r.choice([P, -1, -2 ** 31, 2 ** 31 - 1]) for x in pool["table"][b]]
    elif fault == "sl":
        sl[:3], sl[-1] = [-2, 2 ** 31 - 2, 2 ** 31 - 2], -5
    gpu = to_gpu(pool)
    got = gpu_lib.kv_map(torch.tensor(sl, **I32), torch.tensor(lens, **I32), gpu, page, 100_000)
    torch.cuda.synchronize()
    new, want = R.kv_map(sl, 1, lens, [-1] * B, pool["table"], pool["held"], pool["free"], pool["n_free"][0], page, P, 100_000)
    want["cu_rows"] = [min(x, 2 ** 31 - 1) for x in want["cu_rows"]]
    for k, v in want.items():
        assert got[k].tolist() == v, k
    for k, v in new.items():
        assert gpu[k].tolist() == v, k
    assert any(want["seq_err"]) or (fault, B) == ("spare 60", 130)  # where 60 pages are enough


def test_lengths_advance_in_place(gpu_lib):
    lens = torch.tensor([5, 0, 77], **I32)
    pool = gpu_lib.new_kv_pool(3, 8, 24)
    sl, acc = torch.tensor([2, 3, 0], **I32), torch.tensor([1, -1, 0], **I32)
    out = gpu_lib.new_kv_map_out(3, 8)
    out["base"] = lens
    got = gpu_lib.kv_map(sl, lens, pool, 16, 8, accepted=acc, out=out)
    assert got["base"].tolist() == [7, 0, 78] and got["context"].tolist() == [10, 4, 79] and lens.tolist() == [7, 0, 78]
    assert got["cu_rows"].tolist() == [0, 3, 7, 8] and got["positions"].tolist() == [7, 8, 9, 0, 1, 2, 3, 78]


def test_a_captured_map_follows_its_inputs(gpu_lib):
    """A graph replayed as the sequences grow, with eager work between, against the loop."""
    r = random.Random(9)
    B, W, page, rows = 70, 20, 16, 700
    P = B * W
    lens, pool = state(r, B, W, page, P, 60)
    gpu = to_gpu(pool)
    sl, kv_len, acc = (torch.zeros(B, **I32) for _ in range(3))
    out, ws = gpu_lib.new_kv_map_out(B, rows), gpu_lib.new_kv_map_workspace(B)
    keep = {k: v.clone() for k, v in gpu.items()}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        gpu_lib.kv_map(sl, kv_len, gpu, page, rows, accepted=acc, out=out, workspace=ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gpu_lib.kv_map(sl, kv_len, gpu, page, rows, accepted=acc, out=out, workspace=ws)
    for k, v in keep.items():
        gpu[k].copy_(v)
    accepted = [-1] * B
    for step in range(6):
        drafts = [r.randrange(0, 9) for _ in range(B)]
        for t, x in ((sl, drafts), (kv_len, lens), (acc, accepted)):
            t.copy_(torch.tensor(x, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        pool, want = R.kv_map(drafts, 1, lens, accepted, pool["table"], pool["held"], pool["free"], pool["n_free"][0], page, P, rows)
        for k, v in want.items():
            assert out[k].tolist() == v, (step, k)
        for k, v in pool.items():
            assert gpu[k].tolist() == v, (step, k)
        lens, accepted = want["base"], [r.randrange(0, d + 1) for d in drafts]
