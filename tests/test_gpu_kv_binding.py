"""What the binding refuses of the cache's tensors, and what it tells torch of the memory it writes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def args(lib, **over):
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache = lib.new_kv_cache(12, 16, 2, 64)
    for c in cache:
        c.zero_()
    a = dict(sl=torch.ones(3, **I32), kv_len=torch.zeros(3, **I32), accepted=None, pool=lib.new_kv_pool(3, 4, 12), page=16, rows=6,
             out=None, ws=None, k=k, v=k.clone(), slots=torch.arange(5, **I32), row_err=None,
             q=torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda"), kc=cache[0], vc=cache[1],
             table=torch.zeros(3, 4, **I32), context=torch.full((3,), 5, **I32), cu=torch.tensor([0, 2, 4, 5], **I32), max_rows=2,
             ks=None, vs=None, window=0, scale=None)
    a.update(over)
    return a


def run(lib, name, **over):
    a = args(lib, **over)
    if name == "kv_map":
        return lib.kv_map(a["sl"], a["kv_len"], a["pool"], a["page"], a["rows"], accepted=a["accepted"], out=a["out"], workspace=a["ws"])
    if name == "kv_write":
        return lib.kv_write(a["k"], a["v"], a["slots"], a["kc"], a["vc"], a["ks"], a["vs"], row_err=a["row_err"])
    return lib.kv_attention(a["q"], a["kc"], a["vc"], a["table"], a["context"], a["cu"], a["max_rows"], a["scale"], a["window"],
                            a["ks"], a["vs"], lse=True, out=a["out"], workspace=a["ws"])


def refused(lib, name, text, **over):
    with pytest.raises(lib.DsdeError, match=text):
        run(lib, name, **over)


def test_good_calls_pass(gpu_lib):
    for name in ("kv_map", "kv_write", "kv_attention"):
        run(gpu_lib, name)
    torch.cuda.synchronize()


def test_map_arguments(gpu_lib):
    z = lambda *n, **kw: torch.zeros(*n, **dict(I32, **kw))  # noqa: E731
    refused(gpu_lib, "kv_map", "sl must be torch.int32, got torch.int64", sl=z(3, dtype=torch.int64))
    refused(gpu_lib, "kv_map", "kv_len has 2 elements, needs 3", kv_len=z(2))
    refused(gpu_lib, "kv_map", "accepted must be torch.int32", accepted=z(3, dtype=torch.float32))
    refused(gpu_lib, "kv_map", "kv_len must be contiguous", kv_len=z(6)[::2])
    refused(gpu_lib, "kv_map", "invalid argument", page=24)
    refused(gpu_lib, "kv_map", "size is out of range", page=4096)
    refused(gpu_lib, "kv_map", "size is out of range", rows=-1, out=gpu_lib.new_kv_map_out(3, 1))
    refused(gpu_lib, "kv_map", "slots has 5 elements, needs 6", out=gpu_lib.new_kv_map_out(3, 5))
    refused(gpu_lib, "kv_map", "workspace too small", ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    pool = gpu_lib.new_kv_pool(3, 4, 12)
    refused(gpu_lib, "kv_map", "table must be", pool=dict(pool, table=z(2, 4)))
    refused(gpu_lib, "kv_map", "table has too few dimensions", pool=dict(pool, table=z(12)))
    refused(gpu_lib, "kv_map", "held has 2 elements", pool=dict(pool, held=z(2)))
    refused(gpu_lib, "kv_map", "free must be torch.int32", pool=dict(pool, free=z(12, dtype=torch.int16)))
    refused(gpu_lib, "kv_map", "table must be a GPU tensor", pool=dict(pool, table=z(3, 4, device="cpu")))
    for key in pool:
        with pytest.raises(KeyError):
            run(gpu_lib, "kv_map", pool={k: v for k, v in pool.items() if k != key})
    out = gpu_lib.new_kv_map_out(3, 6)
    for dtype in (torch.uint8, torch.int64, torch.float32):
        refused(gpu_lib, "kv_map", "seq_err must be torch.int32", out=dict(out, seq_err=z(3, dtype=dtype)))


def test_caches(gpu_lib):
    bf16 = torch.bfloat16
    for name in ("kv_write", "kv_attention"):
        def c(*shape, dtype=bf16):
            x = torch.zeros(*shape, dtype=dtype, device="cuda")
            return dict(kc=x, vc=x.clone())
        good = c(12, 2, 16, 64)
        refused(gpu_lib, name, "one type, shape and layout", kc=good["kc"], vc=good["vc"][:11])
        refused(gpu_lib, name, "one type, shape and layout", kc=good["kc"], vc=good["vc"].float())
        refused(gpu_lib, name, "one type, shape and layout", kc=good["kc"], vc=torch.zeros(12, 16, 2, 64, dtype=bf16, device="cuda").transpose(1, 2))
        refused(gpu_lib, name, "bfloat16, float32 or float8_e4m3fn", **c(12, 2, 16, 64, dtype=torch.float16))
        refused(gpu_lib, name, "pages, heads, page_size, dim|too few dimensions", **c(12, 2, 16 * 64))
        refused(gpu_lib, name, "page_size must be", **c(12, 2, 24, 64))
        refused(gpu_lib, name, "page_size must be", **c(12, 2, 8, 64))
        refused(gpu_lib, name, "dim must be a multiple of 16", **c(12, 2, 16, 72))
        refused(gpu_lib, name, "dim must be a multiple of 16", **c(12, 2, 16, 272))
        refused(gpu_lib, name, "dense heads", kc=good["kc"].transpose(2, 3).expand(12, 2, 64, 16)[:, :, :, :16], vc=good["vc"])
        refused(gpu_lib, name, "multiples of 16 bytes", **{k: torch.zeros(12, 2, 16, 68, dtype=bf16, device="cuda")[..., :64] for k in ("kc", "vc")})
        refused(gpu_lib, name, "k_scale and v_scale belong", ks=torch.ones(2, device="cuda"), vs=torch.ones(2, device="cuda"))
        e4m3 = c(12, 2, 16, 64, dtype=torch.float8_e4m3fn)
        refused(gpu_lib, name, "k_scale and v_scale belong", **e4m3)
        refused(gpu_lib, name, "k_scale has 1 elements", **e4m3, ks=torch.ones(1, device="cuda"), vs=torch.ones(2, device="cuda"))
        run(gpu_lib, name, **e4m3, ks=torch.ones(2, device="cuda"), vs=torch.ones(2, device="cuda"))
    over = torch.zeros(1, 2, 16, 64, dtype=bf16, device="cuda").expand(12, -1, -1, -1)
    refused(gpu_lib, "kv_write", "invalid argument", kc=over, vc=over)  # pages that are one


def test_rows(gpu_lib):
    z = lambda *n, dtype=torch.bfloat16: torch.zeros(*n, dtype=dtype, device="cuda")  # noqa: E731
    refused(gpu_lib, "kv_write", "k must have the cache's dim", k=z(5, 2, 48))
    refused(gpu_lib, "kv_write", "of the cache's type", k=z(5, 2, 64, dtype=torch.float32))
    refused(gpu_lib, "kv_write", "of the cache's heads", k=z(5, 3, 64), v=z(5, 3, 64))
    refused(gpu_lib, "kv_write", "of the cache's heads", v=z(4, 2, 64))
    refused(gpu_lib, "kv_write", "slots has 4 elements", slots=torch.zeros(4, **I32))
    refused(gpu_lib, "kv_write", "dense heads", k=z(5, 2, 128)[:, :, ::2])
    refused(gpu_lib, "kv_write", "multiples of 16 bytes", k=z(5, 2, 65)[:, :, 1:])
    refused(gpu_lib, "kv_write", "row_err must be torch.int32", row_err=z(5))
    refused(gpu_lib, "kv_attention", "multiple of the cache's heads", q=z(5, 3, 64))
    refused(gpu_lib, "kv_attention", "q must have the cache's dim", q=z(5, 4, 128))
    refused(gpu_lib, "kv_attention", "of the cache's type", q=z(5, 4, 64, dtype=torch.float32))
    refused(gpu_lib, "kv_attention", "context has 2 elements", context=torch.zeros(2, **I32))
    refused(gpu_lib, "kv_attention", "cu_rows has 3 elements", cu=torch.zeros(3, **I32))
    refused(gpu_lib, "kv_attention", "table must be torch.int32", table=torch.zeros(3, 4, device="cuda"))
    refused(gpu_lib, "kv_attention", "table must be contiguous", table=torch.zeros(3, 8, **I32)[:, ::2])
    refused(gpu_lib, "kv_attention", "invalid sizes", max_rows=65)
    refused(gpu_lib, "kv_attention", "window must be", window=-1)
    refused(gpu_lib, "kv_attention", "window must be", window=1 << 31)
    refused(gpu_lib, "kv_attention", "invalid argument", scale=float("nan"))
    out = run(gpu_lib, "kv_attention")
    refused(gpu_lib, "kv_attention", "out must have the queries' shape", out=dict(out, out=z(5, 4, 48)))
    refused(gpu_lib, "kv_attention", "out must have the queries' shape", out=dict(out, out=z(5, 4, 64, dtype=torch.float32)))
    refused(gpu_lib, "kv_attention", "lse has 4 elements", out=dict(out, lse=torch.zeros(4, device="cuda")))
    refused(gpu_lib, "kv_attention", "seq_err must be torch.int32", out=dict(out, seq_err=z(3)))
    refused(gpu_lib, "kv_attention", "invalid argument", out=dict(out, out=z(1, 4, 64).expand(5, 4, 64)))
    refused(gpu_lib, "kv_attention", "workspace too small", ws=torch.empty(64, dtype=torch.uint8, device="cuda"))


def test_writes_raise_versions(gpu_lib):
    a = args(gpu_lib)
    out = gpu_lib.kv_map(a["sl"], a["kv_len"], a["pool"], 16, 6)
    written = dict(out, **a["pool"])
    before = {k: v._version for k, v in written.items()}
    gpu_lib.kv_map(a["sl"], a["kv_len"], a["pool"], 16, 6, out=out)
    assert all(v._version > before[k] for k, v in written.items()) and a["sl"]._version == a["kv_len"]._version == 0
    out = gpu_lib.kv_attention(a["q"], a["kc"], a["vc"], a["table"], a["context"], a["cu"], 2, lse=True)
    before = {k: v._version for k, v in out.items()}
    version = a["kc"]._version
    gpu_lib.kv_attention(a["q"], a["kc"], a["vc"], a["table"], a["context"], a["cu"], 2, out=out)
    assert all(v._version > before[k] for k, v in out.items()) and a["kc"]._version == version and a["q"]._version == 0
    with torch.inference_mode():
        got = run(gpu_lib, "kv_attention")
        run(gpu_lib, "kv_write")
    run(gpu_lib, "kv_attention", out=got)
