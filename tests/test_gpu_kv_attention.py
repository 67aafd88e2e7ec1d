"""dsde_kv_attention against its definition in 64 bits, within bounds that count the roundings."""
import math

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -8}
NAN = float("nan")


def make(context, n, H=2, G=2, D=64, S=16, dtype="bf16", by_token=False, seed=0, junk=True, strength=1.0, extra_width=2):
    """Inputs on the CPU; what no sequence holds is NaN, infinite or huge."""
    g = torch.Generator().manual_seed(seed)
    P = sum(-(-c // S) for c in context) + 3
    pages = R.pages_of(context, S, P, seed)
    width = max(max(len(x) for x in pages), 1) + extra_width
    row_dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    q = (strength * torch.randn(sum(n), H * G, D, generator=g)).to(row_dt)
    kv = []
    for _ in range(2):
        x = torch.randn(P, H, S, D, generator=g).to(DT[dtype])
        if junk:
            used = torch.zeros(P, S, dtype=torch.bool)
            for c, ids in zip(context, pages):
                for i, p in enumerate(ids):
                    used[p, :min(S, c - i * S)] = True
            bad = torch.tensor([NAN, math.inf, -math.inf, 3e38]).to(DT[dtype])[torch.randint(0, 4, (P, H, S, D), generator=g)]
            raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
            x = torch.where(used[:, None, :, None], x.view(raw), bad.view(raw)).view(DT[dtype])
        kv.append(x)
    scales = [0.5 + torch.rand(H, generator=g) if dtype == "e4m3" else None for _ in range(2)]
    return dict(q=q, k=kv[0], v=kv[1], k_scale=scales[0], v_scale=scales[1], table=R.table_of(pages, width),
                context=list(context), cu=R.prefix(n), max_rows=max(max(n), 1), by_token=by_token, dtype=dtype)


def to_gpu(x):
    def layout(c):
        c = c.cuda()
        return c.transpose(1, 2).contiguous().transpose(1, 2) if x["by_token"] else c
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(q=x["q"].cuda(), k_cache=layout(x["k"]), v_cache=layout(x["v"]), table=x["table"].cuda(),
                context=torch.tensor(x["context"], **i32), cu_rows=torch.tensor(x["cu"], **i32), max_rows=x["max_rows"],
                k_scale=None if x["k_scale"] is None else x["k_scale"].cuda(),
                v_scale=None if x["v_scale"] is None else x["v_scale"].cuda())


def compare(x, got, scale=None, window=0):
    D = x["q"].shape[2]
    out, lse, e_out, e_lse = R.attend(x["q"], x["k"], x["v"], x["table"], x["context"], x["cu"],
                                      D ** -0.5 if scale is None else scale, window, x["k_scale"], x["v_scale"], EPS[x["dtype"]])
    o, z = got["out"].cpu().double(), got["lse"].cpu().double()
    empty = lse == -math.inf
    assert torch.equal(z == -math.inf, empty)
    assert bool((o[empty] == 0).all())
    d = (o - out).abs()
    assert bool((d <= e_out).all()), (float((d / e_out.clamp(min=1e-30)).max()), float(d.max()))
    d = (z - lse).masked_fill(empty, 0.0).abs()
    assert bool((d <= e_lse).all()), (float((d / e_lse.clamp(min=1e-30)).max()), float(d.max()))
    assert not got["seq_err"].any()


def check(lib, x, scale=None, window=0, **kw):
    print(x["q"].shape, x["k"].shape, x["context"], x["cu"], window, flush=True)
    got = lib.kv_attention(**to_gpu(x), scale=scale, window=window, lse=True, **kw)
    torch.cuda.synchronize()
    compare(x, got, scale, window)
    return got


TYPES = ["bf16", "fp32", "e4m3"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128, 160, 192, 208, 256])
def test_head_sizes(gpu_lib, D, dtype):
    check(gpu_lib, make([1, 15, 40, 130], [1, 1, 1, 1], D=D, dtype=dtype, seed=D))
    check(gpu_lib, make([70, 3], [5, 2], H=1, G=4, D=D, dtype=dtype, seed=D + 1, by_token=True))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S", [16, 32, 64, 128, 256, 512, 1024])
def test_page_sizes_and_lengths(gpu_lib, S, dtype):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 600]
    check(gpu_lib, make(lens, [1] * len(lens), S=S, dtype=dtype, seed=S))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,G", [(1, 1), (1, 16), (1, 17), (3, 5), (2, 7), (8, 4), (1, 32), (1, 64), (12, 1), (1, 71), (5, 3)])
def test_head_layouts(gpu_lib, H, G, dtype):
    check(gpu_lib, make([50, 333, 7], [1, 1, 1], H=H, G=G, dtype=dtype, seed=H * G))
    check(gpu_lib, make([50, 120, 7], [3, 9, 2], H=H, G=G, dtype=dtype, seed=H * G))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [2, 4, 9, 17, 33, 64])
def test_rows_of_a_step(gpu_lib, n, dtype):
    """SL + 1 rows each: ragged, with sequences of one row and of none."""
    lens = [n, n + 1, 40 + n, 100, 5, 64, 200]
    rows = [n, n, max(1, n // 2), 0, 1, min(n, 64), n]
    check(gpu_lib, make(lens, rows, G=2, dtype=dtype, seed=n))
    check(gpu_lib, make(lens, rows, H=1, G=8, D=128, dtype=dtype, seed=n))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,G,most", [(64, 4, 8), (128, 4, 8), (64, 5, 9), (64, 7, 9)])
def test_row_blocks_that_come_and_go(gpu_lib, D, G, most, dtype):
    """Wavefronts that go from items with few rows to items with many, and back."""
    g = torch.Generator().manual_seed(G * D)
    lens = torch.randint(1, 120, (280,), generator=g).tolist()
    n = torch.randint(0, most + 1, (280,), generator=g).tolist()
    check(gpu_lib, make(lens, n, H=3, G=G, D=D, dtype=dtype, seed=G * D))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 31, 33, 64, 100, 1000])
def test_windows(gpu_lib, window, dtype):
    check(gpu_lib, make([1, 16, 33, 150, 400], [1, 4, 9, 3, 5], dtype=dtype, seed=window), window=window)
    check(gpu_lib, make([300, 90], [1, 1], H=1, G=8, D=128, S=64, dtype=dtype, seed=window), window=window)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_see_nothing(gpu_lib, dtype):
    """Contexts shorter than the rows, and of no token at all."""
    check(gpu_lib, make([0, 2, 0, 5, 64], [3, 5, 1, 9, 2], dtype=dtype))
    check(gpu_lib, make([0], [1], dtype=dtype))
    check(gpu_lib, make([0, 0], [0, 0], dtype=dtype, extra_width=1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,most", [(1, 5000), (3, 2500), (40, 300), (700, 40)])
def test_split_and_joined(gpu_lib, B, most, dtype):
    """Long caches over many workgroups, and many short ones in one."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(max(1, most // 3), most + 1, (B,), generator=g).tolist()
    n = torch.randint(0, 3, (B,), generator=g).tolist()
    n[0] = 1
    check(gpu_lib, make(lens, n, H=1 if B > 1 else 2, G=2, D=64, dtype=dtype, seed=B))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("strength,scale", [(30.0, None), (1.0, 0.0), (1.0, -0.3), (1e-3, 7.0), (200.0, None)])
def test_scores_of_any_size(gpu_lib, strength, scale, dtype):
    """One token with all weight, equal weights, references that rise late."""
    x = make([700, 45, 130], [1, 3, 2], dtype=dtype, strength=strength)
    order = torch.argsort((x["k"].float().nan_to_num(0, 0, 0) ** 2).sum((1, 2, 3)))  # noqa: F841 (any order is fine)
    check(gpu_lib, x, scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_ascending_scores(gpu_lib, dtype):
    """Every tile raises the reference, by little and by much."""
    for slope in (0.01, 0.3, 4.0):
        x = make([900], [1], H=1, G=1, D=64, dtype=dtype, junk=False)
        x["q"].zero_()
        x["q"][0, 0, 0] = 1.0
        ids = x["table"][0, :57].long()
        k = x["k"].float()
        t = torch.arange(57 * 16).view(57, 16) * slope
        k[ids, 0, :, 0] = t if dtype != "e4m3" else t.clamp(max=448)
        x["k"] = k.to(DT[dtype])
        check(gpu_lib, x, scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("what", [NAN, math.inf])
def test_values_that_some_rows_see(gpu_lib, dtype, what):
    """A NaN or infinite value of a drafted token: rows before it are unharmed, rows from it on have it."""
    what = NAN if dtype == "e4m3" else what
    for n, c, at, window in ((5, 70, 67, 0), (9, 40, 35, 0), (4, 100, 20, 78), (33, 64, 40, 0)):
        x = make([c], [n], H=1, G=2, D=64, dtype=dtype)
        clean = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in x.items()}
        page, i = int(x["table"][0, at // 16]), at % 16
        x["v"][page, 0, i, 7] = what
        got = gpu_lib.kv_attention(**to_gpu(x), window=window, lse=True)
        want = gpu_lib.kv_attention(**to_gpu(clean), window=window, lse=True)
        assert torch.equal(got["lse"], want["lse"])
        for j in range(n):
            p = c - n + j
            sees = at <= p and (window == 0 or at > p - window)
            o = got["out"][j].float().cpu()
            assert bool((~torch.isfinite(o[:, 7])).all()) == sees, (n, j)
            rest = torch.ones(64, dtype=torch.bool)
            rest[7] = not sees
            assert torch.equal(o[:, rest], want["out"][j].float().cpu()[:, rest]), (n, j)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_keys_that_are_not_finite(gpu_lib, dtype):
    """A key of -inf for a positive query: weight 0; a NaN key: its rows are NaN."""
    x = make([40], [2], H=1, G=1, D=64, dtype=dtype)
    x["q"][:, 0, 3] = 1.0
    x["k"][int(x["table"][0, 0]), 0, 4, 3] = -math.inf
    check(gpu_lib, x)
    x["k"][int(x["table"][0, 2]), 0, 7, 3] = NAN  # token 39: the second row's own
    got = gpu_lib.kv_attention(**to_gpu(x), lse=True)
    assert bool(torch.isfinite(got["out"][0]).all()) and bool(torch.isnan(got["out"][1]).all()) and bool(torch.isnan(got["lse"][1]).all())


def test_layouts_of_rows_and_caches(gpu_lib):
    """Queries cut out of a wider projection, outputs into one, one page of a larger cache."""
    x = make([60, 33], [4, 1], H=2, G=3, D=48)
    y = to_gpu(x)
    want = gpu_lib.kv_attention(**y, lse=True)
    wide = torch.full((5, 2, 6, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 0, :, :48] = y["q"]
    out = dict(out=wide[:, 1, :, :48], lse=torch.empty(5, 6, device="cuda"), seq_err=torch.empty(2, dtype=torch.int32, device="cuda"))
    caches = torch.full((y["k_cache"].shape[0], 2, 4, 16, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    caches[:, 0, 1:3, :, :48], caches[:, 1, 1:3, :, :48] = y["k_cache"], y["v_cache"]
    z = dict(y, q=wide[:, 0, :, :48], k_cache=caches[:, 0, 1:3, :, :48], v_cache=caches[:, 1, 1:3, :, :48])
    got = gpu_lib.kv_attention(**z, out=out)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    assert bool((wide[:, 1, :, 48:] == 5).all()) and torch.equal(wide[:, 0, :, :48], y["q"])


def test_rows_of_no_sequence_are_left(gpu_lib):
    x = make([20, 40], [2, 1], H=1, G=2)
    y = to_gpu(x)
    want = gpu_lib.kv_attention(**y, lse=True)
    q = torch.cat([torch.ones_like(y["q"][:4]), y["q"], torch.ones_like(y["q"])])[1:]
    out = dict(out=torch.full_like(q, 3.0), lse=torch.full(q.shape[:2], 4.0, device="cuda"),
               seq_err=torch.empty(2, dtype=torch.int32, device="cuda"))
    cu = y["cu_rows"] + 2  # the first rows belong to no sequence either
    got = gpu_lib.kv_attention(**dict(y, q=q, cu_rows=cu), out=out)
    assert torch.equal(got["out"][2:5], want["out"]) and torch.equal(got["lse"][2:5], want["lse"])
    rest = [0, 1] + list(range(5, len(q)))
    assert bool((got["out"][rest] == 3).all()) and bool((got["lse"][rest] == 4).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_faults_are_flagged(gpu_lib, dtype):
    """Bad pages, contexts and rows, each in a sequence of its own between sound ones."""
    x = make([50, 50, 50, 50, 50, 50, 50], [2, 2, 2, 2, 2, 2, 2], H=2, G=2, dtype=dtype, junk=False)
    y = to_gpu(x)
    want = gpu_lib.kv_attention(**y, lse=True)
    P = x["k"].shape[0]
    y["table"][1, 1], y["table"][2, 3], y["table"][3, 0] = -1, P, 2 ** 31 - 1
    y["context"][4], y["context"][5] = -3, 16 * y["table"].shape[1] + 1
    got = gpu_lib.kv_attention(**y, lse=True)
    assert got["seq_err"].tolist() == [0, 256, 256, 256, 1, 1, 0]
    for b in range(7):
        o, z = got["out"][2 * b:2 * b + 2], got["lse"][2 * b:2 * b + 2]
        if b in (0, 6):
            assert torch.equal(o, want["out"][2 * b:2 * b + 2]) and torch.equal(z, want["lse"][2 * b:2 * b + 2])
        elif b == 2:  # token 48, the first row's own, is in the bad page
            assert bool(torch.isnan(o).all()) and bool(torch.isnan(z).all())
        else:
            assert bool(torch.isnan(o).all()) and bool(torch.isnan(z).all())
    # a window that does not reach the bad page
    got = gpu_lib.kv_attention(**y, lse=True, window=10)
    assert got["seq_err"].tolist() == [0, 0, 256, 0, 1, 1, 0]
    y = to_gpu(x)
    y["cu_rows"] = torch.tensor([0, 2, 1, 6, 8, 10, 12, 99], dtype=torch.int32, device="cuda")
    got = gpu_lib.kv_attention(**dict(y, max_rows=4), lse=True)
    assert got["seq_err"].tolist() == [0, 1, 1, 0, 0, 0, 1]
    assert torch.equal(got["out"][8:12], want["out"][8:12])
    y["cu_rows"] = torch.tensor([-2, 0, 2, 4, 6, 8, 10, 12], dtype=torch.int32, device="cuda")
    got = gpu_lib.kv_attention(**y)
    assert got["seq_err"].tolist() == [1, 0, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_before_a_bad_page_are_unharmed(gpu_lib, dtype):
    """Rows of tokens 44 .. 52, the page of 48 on bad: those before it are as they were, in one head's item and in parts."""
    for c, n, bad in ((53, 9, 3), (2003, 9, 125), (700, 33, 42)):
        x = make([c], [n], H=1, G=2, D=64, dtype=dtype, junk=False)
        y = to_gpu(x)
        want = gpu_lib.kv_attention(**y, lse=True)
        for page in (-1, x["k"].shape[0]):
            y["table"][0, bad] = page
            got = gpu_lib.kv_attention(**y, lse=True)
            assert got["seq_err"].tolist() == [256]
            for j in range(n):
                if c - n + j >= 16 * bad:
                    assert bool(torch.isnan(got["out"][j]).all()) and bool(torch.isnan(got["lse"][j]).all()), j
                else:
                    assert torch.equal(got["out"][j], want["out"][j]) and torch.equal(got["lse"][j], want["lse"][j]), j


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_values_of_both_signs(gpu_lib, dtype):
    """+inf, then -inf in one dimension: inf, then NaN; alone in others; in the last tile of a long cache too."""
    for c in (64, 1500):
        x = make([c], [4], H=2, G=3, D=128, dtype=dtype, junk=False)
        for at, d, value in ((c - 3, 5, math.inf), (c - 2, 5, -math.inf), (c - 2, 100, -math.inf), (c - 1, 64, math.inf)):
            x["v"][int(x["table"][0, at // 16]), 1, at % 16, d] = value
        o = gpu_lib.kv_attention(**to_gpu(x))["out"][:, 3:].float().cpu()  # the second key head's
        assert bool(torch.isfinite(o[0]).all())
        assert bool((o[1, :, 5] == math.inf).all()) and bool(torch.isnan(o[2:, :, 5]).all())
        assert bool((o[2:, :, 100] == -math.inf).all()) and bool((o[3, :, 64] == math.inf).all())
        o[:, :, [5, 64, 100]] = 0
        assert bool(torch.isfinite(o).all())


def test_one_page_for_many(gpu_lib):
    """Sequences that share pages, and one whose table is the same page throughout: 2^20 tokens of a cache of 64."""
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(4, 1, 16, 16, generator=g) for _ in range(2))
    n = 1 << 16
    table = torch.zeros(2, n, dtype=torch.int32)
    table[1] = torch.arange(n) % 4
    q = torch.randn(2, 1, 16, generator=g)
    i32 = dict(dtype=torch.int32, device="cuda")
    got = gpu_lib.kv_attention(q.cuda(), k.cuda(), v.cuda(), table.cuda(), torch.tensor([16 * n, 16 * n], **i32),
                               torch.tensor([0, 1, 2], **i32), 1, lse=True)
    for b, (kk, vv, times) in enumerate(((k[0, 0], v[0, 0], n), (k[:, 0].reshape(64, 16), v[:, 0].reshape(64, 16), n // 4))):
        z = kk.double() @ q[b, 0].double() / 4
        want = torch.softmax(z, 0) @ vv.double()
        # sums of 2^20 weights: 2^20 / 64 of a lane in a row at most 2^14 2^-24 off, of values of size sum p |v|
        A = torch.softmax(z, 0) @ vv.double().abs()
        assert bool(((got["out"][b, 0].cpu().double() - want).abs() <= 2.0 ** -10 * A).all())
        lse = torch.logsumexp(z, 0) + math.log(times)
        assert abs(float(got["lse"][b, 0]) - float(lse)) <= 2.0 ** -10
    assert not got["seq_err"].any()


def test_calls_repeat_bit_for_bit(gpu_lib):
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(1, 900, (50,), generator=g).tolist()
    y = to_gpu(make(lens, [3] * 50, H=4, G=4, D=128))
    first = gpu_lib.kv_attention(**y, lse=True)
    ws = gpu_lib.new_kv_attention_workspace(50, 4, 4, 3, 128)
    for fill in (0, 255, 127):
        ws.fill_(fill)
        again = gpu_lib.kv_attention(**y, lse=True, workspace=ws)
        assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])


def test_streams_and_graphs(gpu_lib):
    """Two captured calls that share a workspace, replayed in turn with eager work between them."""
    a, b = to_gpu(make([500, 30, 222], [2, 3, 1], seed=1)), to_gpu(make([64, 700], [1, 4], seed=2))
    want = [gpu_lib.kv_attention(**y, lse=True) for y in (a, b)]
    ws = gpu_lib.new_kv_attention_workspace(3, 2, 2, 4, 64)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for y, w in zip((a, b), want):
        out = {k: torch.empty_like(v) for k, v in w.items()}
        gpu_lib.kv_attention(**y, out=out, workspace=ws, stream=side)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            gpu_lib.kv_attention(**y, out=out, workspace=ws)
        graphs.append(g)
        outs.append(out)
    for _ in range(4):
        for g, out, w, y in zip(graphs, outs, want, (a, b)):
            for v in out.values():
                v.fill_(9)
            g.replay()
            again = gpu_lib.kv_attention(**y, lse=True)
            torch.cuda.synchronize()
            for k in w:
                assert torch.equal(out[k], w[k]) and torch.equal(again[k], w[k]), k
