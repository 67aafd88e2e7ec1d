"""Host-side checks of the paged cache's calls (no GPU needed): what the C ABI and the
binding refuse, workspace sizes, and whose stream a call's own buffers belong to."""
import ctypes

import pytest
import torch

from test_binding_host import FakeNative, FakeStream, RawStream, Recorder

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1008)


@pytest.fixture(scope="module")
def dsde():
    import paper_2509_01083_amd as dsde
    dsde._bind()
    return dsde


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


GOOD = dict(k=0x1000, v=0x2000, dtype=1, pages=100, page_size=16, heads=8, dim=128, page_stride=16384, head_stride=2048,
            token_stride=128, k_scale=None, v_scale=None)
BAD_CACHES = [dict(k=None), dict(v=None), dict(dtype=3), dict(dtype=-1), dict(pages=0), dict(pages=1 << 27), dict(page_size=15),
              dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(heads=0), dict(heads=1025), dict(dim=0),
              dict(dim=8), dict(dim=120), dict(dim=272), dict(page_stride=-16384), dict(head_stride=-2048),
              dict(token_stride=-128), dict(page_stride=16383), dict(head_stride=2049), dict(token_stride=132),
              dict(page_stride=16376), dict(head_stride=64), dict(token_stride=64), dict(head_stride=2040),
              dict(page_stride=8 * 2048 - 128), dict(k=0x1008), dict(v=0x2004), dict(dtype=2), dict(dtype=2, k_scale=0x1000),
              dict(k_scale=0x1000, v_scale=0x1000), dict(page_stride=1 << 41), dict(token_stride=1 << 34, page_stride=1 << 39)]
MAP = dict(B=4, page_size=16, pages=100, width=10, rows=50, sl=FAKE, extra=1, kv_len=FAKE, accepted=None, table=FAKE, held=FAKE,
           free=FAKE, n_free=FAKE, base=FAKE, context=FAKE, cu=FAKE, slots=FAKE, positions=FAKE, err=FAKE, ws=FAKE,
           ws_bytes=1 << 30, stream=None)
WRITE = dict(cache=None, k=FAKE, k_token=1024, k_head=128, v=FAKE, v_token=1024, v_head=128, dtype=1, T=3, slots=FAKE, err=FAKE,
             stream=None)
ATTEND = dict(cache=None, q=FAKE, q_token=4096, q_head=128, dtype=1, q_heads=32, T=3, B=2, max_rows=4, table=FAKE, width=10,
              context=FAKE, cu=FAKE, scale=1.0, window=0, out=FAKE, out_token=4096, out_head=128, lse=None, err=FAKE, ws=FAKE,
              ws_bytes=1 << 30, stream=None)


def rc(dsde, name, args, cache=None):
    args = dict(args)
    if "cache" in args and args["cache"] is None:
        args["cache"] = ctypes.byref(Cache(**dict(GOOD, **(cache or {}))))
    return getattr(dsde.load(), name)(*args.values())


def test_map_refuses(dsde):
    bad = [dict(B=0), dict(B=-1), dict(B=(1 << 20) + 1), dict(page_size=0), dict(page_size=24), dict(page_size=2048), dict(pages=0),
           dict(pages=1 << 27), dict(width=0), dict(width=1 << 27), dict(width=(1 << 26) + 1), dict(rows=-1), dict(rows=1 << 31), dict(ws=ODD)]
    bad += [{k: None} for k, v in MAP.items() if isinstance(v, ctypes.c_void_p)]
    for over in bad:
        assert rc(dsde, "dsde_kv_map", dict(MAP, **over)) == 1, over
    assert rc(dsde, "dsde_kv_map", dict(MAP, ws_bytes=64)) == 2


@pytest.mark.parametrize("name,args", [("dsde_kv_write", WRITE), ("dsde_kv_attention", ATTEND)])
def test_caches_are_refused(dsde, name, args):
    for over in BAD_CACHES:
        assert rc(dsde, name, args, over) == 1, over
    assert getattr(dsde.load(), name)(*dict(args, cache=None).values()) == 1


def test_write_refuses(dsde):
    bad = [dict(dtype=0), dict(dtype=2), dict(dtype=5), dict(T=-1), dict(T=1 << 31), dict(k=None), dict(v=None), dict(slots=None),
           dict(err=None), dict(k=ODD), dict(v=ODD), dict(k_token=1023), dict(v_head=124), dict(k_token=-1024), dict(v_token=1 << 41)]
    for over in bad:
        assert rc(dsde, "dsde_kv_write", dict(WRITE, **over)) == 1, over
    e4m3 = dict(dtype=2, k_scale=0x1000, v_scale=0x1000)
    assert rc(dsde, "dsde_kv_write", dict(WRITE, dtype=0), e4m3) == 1
    assert rc(dsde, "dsde_kv_write", WRITE, dict(v=GOOD["k"])) == 1  # keys and values in one place
    none = dict(WRITE, T=0, k=None, v=None, slots=None, err=None)
    assert rc(dsde, "dsde_kv_write", none) == 0 and rc(dsde, "dsde_kv_write", none, e4m3) == 0


def test_attention_refuses(dsde):
    bad = [dict(dtype=0), dict(dtype=2), dict(q_heads=0), dict(q_heads=12), dict(q_heads=1032), dict(T=-1), dict(T=1 << 31),
           dict(B=0), dict(B=(1 << 20) + 1), dict(max_rows=0), dict(max_rows=65), dict(width=0), dict(width=1 << 27),
           dict(width=(1 << 26) + 1), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(scale=-2.4e38), dict(window=-1), dict(q=ODD), dict(out=ODD), dict(ws=ODD),
           dict(q_token=4097), dict(q_head=-128), dict(out_token=4100), dict(out_token=2048), dict(out_head=64), dict(out_head=0)]
    bad += [{k: None} for k, v in ATTEND.items() if isinstance(v, ctypes.c_void_p)]
    for over in bad:
        assert rc(dsde, "dsde_kv_attention", dict(ATTEND, **over)) == 1, over
    assert rc(dsde, "dsde_kv_attention", dict(ATTEND, ws_bytes=1024)) == 2


def test_workspace_sizes(dsde):
    lib = dsde.load()
    for bad in (0, -1, (1 << 20) + 1):
        assert lib.dsde_kv_map_workspace_bytes(bad) == 0
    sizes = [lib.dsde_kv_map_workspace_bytes(B) for B in (1, 2, 64, 1000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    ws = lib.dsde_kv_attention_workspace_bytes
    good = dict(B=4, heads=8, group=4, max_rows=9, dim=128)
    for over in (dict(B=0), dict(B=(1 << 20) + 1), dict(heads=0), dict(heads=1025), dict(group=0), dict(group=129),
                 dict(max_rows=0), dict(max_rows=65), dict(dim=0), dict(dim=24), dict(dim=272), dict(group=(1 << 31) - 1)):
        assert ws(*dict(good, **over).values()) == 0, over
    grows = dict(B=[1, 2, 300, 1 << 20], heads=[1, 2, 8], group=[1, 2, 3, 16, 17, 100], max_rows=[1, 2, 5, 9, 64],
                 dim=[16, 64, 80, 128, 144, 192, 256])
    for k, values in grows.items():
        for base in (good, dict(good, group=1, max_rows=1, dim=16), dict(good, max_rows=64, dim=256, group=16)):
            sizes = [ws(*dict(base, **{k: v}).values()) for v in values]
            assert sizes == sorted(sizes) and sizes[0] > 0, (k, sizes)


def calls(dsde, stream=None, **over):
    """Every call on CPU tensors, as name -> function."""
    i32 = dict(dtype=torch.int32)
    a = dict(sl=torch.zeros(3, **i32), kv_len=torch.zeros(3, **i32), pool=dsde.new_kv_pool(3, 4, 12, device="cpu"), page=16, rows=5,
             k=torch.zeros(5, 2, 64, dtype=torch.bfloat16), v=torch.zeros(5, 2, 64, dtype=torch.bfloat16),
             slots=torch.zeros(5, **i32), q=torch.zeros(5, 4, 64, dtype=torch.bfloat16),
             cache=dsde.new_kv_cache(12, 16, 2, 64, device="cpu"), table=torch.zeros(3, 4, **i32), context=torch.zeros(3, **i32),
             cu=torch.zeros(4, **i32), scale=(None, None), window=0)
    a.update(over)
    return {
        "kv_map": lambda: dsde.kv_map(a["sl"], a["kv_len"], a["pool"], a["page"], a["rows"], stream=stream),
        "kv_write": lambda: dsde.kv_write(a["k"], a["v"], a["slots"], *a["cache"], *a["scale"], stream=stream),
        "kv_attention": lambda: dsde.kv_attention(a["q"], *a["cache"], a["table"], a["context"], a["cu"], 2, window=a["window"],
                                                  k_scale=a["scale"][0], v_scale=a["scale"][1], lse=True, stream=stream),
    }


def refused(dsde, name, text, **over):
    with pytest.raises(dsde.DsdeError, match=text):
        calls(dsde, **over)[name]()


def test_cpu_tensors_are_refused(dsde):
    refused(dsde, "kv_map", "sl must be a GPU tensor")
    refused(dsde, "kv_write", "k must be a GPU tensor")
    refused(dsde, "kv_attention", "q must be a GPU tensor")
    refused(dsde, "kv_write", "k must be a GPU tensor", k=None)
    refused(dsde, "kv_map", "sl must be a GPU tensor", sl=None)
    refused(dsde, "kv_attention", "q must be a GPU tensor", q=None)
    refused(dsde, "kv_attention", "table must be a GPU tensor", table=[1])
    refused(dsde, "kv_attention", "k_cache must be a GPU tensor", cache=(None, None))


def test_rows_are_refused(dsde):
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for bad, text in ((k.half(), "bfloat16 or float32"), (k.double(), "bfloat16 or float32"), (k[0], "few dimensions"),
                      (k[None], "rows, heads, dim")):
        refused(dsde, "kv_write", text, k=bad)
    for bad, text in ((k.half(), "bfloat16 or float32"), (k[0], "rows, heads, dim"), (k[None], "rows, heads, dim")):
        refused(dsde, "kv_attention", text, q=bad)


@pytest.mark.parametrize("stream", [None, FakeStream(), RawStream()])
def test_own_buffers_belong_to_the_calls_stream(dsde, monkeypatch, stream):
    stack = ["current"]

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            stack.append(self.s)

        def __exit__(self, *exc):
            stack.pop()

    run = calls(dsde, stream=stream)
    monkeypatch.setattr(dsde, "_native", FakeNative())
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "Stream", FakeStream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
    want = "current" if stream is None else 78 if isinstance(stream, RawStream) else stream
    made = dict(kv_map=7, kv_write=1, kv_attention=4)
    for name, f in run.items():
        with Recorder(stack) as seen:
            f()
        assert seen.seen == [want] * made[name], name
