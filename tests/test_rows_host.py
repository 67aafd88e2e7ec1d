"""Host-side checks of the row operators (no GPU needed): what the C ABI and the
binding refuse, and whose stream a call's own buffers belong to."""
import ctypes

import pytest
import torch

from test_binding_host import FakeNative, FakeStream, RawStream, Recorder

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def dsde():
    import paper_2509_01083_amd as dsde
    dsde._bind()
    return dsde


ROWS = dict(logits=FAKE, stride=1000, dtype=1, V=1000, R=4)
SAMPLE = dict(ROWS, T=FAKE, k=FAKE, p=FAKE, m=FAKE, u=FAKE, pad=-1, tokens=FAKE, logprob=None, kept=None, err=FAKE,
              ws=FAKE, ws_bytes=1 << 30, stream=None)
TOP = dict(ROWS, k=8, T=1.0, values=FAKE, ids=FAKE, lse=FAKE, err=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
LOSS = dict(ROWS, K=8, ids=FAKE, teacher=FAKE, lse=None, T=1.0, loss=FAKE, record=FAKE, err=FAKE, ws=FAKE,
            ws_bytes=1 << 30, stream=None)
GRAD = dict(ROWS, K=8, ids=FAKE, teacher=FAKE, T=1.0, record=FAKE, weight=FAKE, grad=ctypes.c_void_p(0x9000),
            grad_stride=1000, stream=None)
STEP = dict(ROWS, K=8, ids=FAKE, teacher=FAKE, lse=None, T=1.0, weight=FAKE, loss=FAKE, grad=ctypes.c_void_p(0x9000),
            grad_stride=1000, err=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
CALLS = dict(dsde_sample=SAMPLE, dsde_top_logits=TOP, dsde_distill_loss=LOSS, dsde_distill_grad=GRAD,
             dsde_distill_step=STEP)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_invalid_arguments(dsde, name):
    lib, args = dsde.load(), CALLS[name]
    bad = [dict(dtype=2), dict(dtype=-1), dict(V=0), dict(V=4194305), dict(R=-1), dict(stride=999), dict(stride=-1),
           dict(R=1 << 31), dict(R=(1 << 31) - 1, V=9000, stride=9000), dict(stride=1 << 41)]
    bad += [{k: None} for k, v in args.items() if isinstance(v, ctypes.c_void_p)
            and k not in (("k", "p", "m") if name == "dsde_sample" else ())]
    if "K" in args:
        bad += [dict(K=0), dict(K=257)]
    if name == "dsde_top_logits":
        bad += [dict(k=0), dict(k=257)]
    if not isinstance(args.get("T"), ctypes.c_void_p):
        bad += [dict(T=x) for x in (0.0, -1.0, 1e6, 1e-6, float("nan"), float("inf"))]
    if "ws" in args:
        bad += [dict(ws=ctypes.c_void_p(0x1001))]
    if "grad" in args:
        bad += [dict(grad_stride=999), dict(grad=FAKE, grad_stride=1001)]
    for over in bad:
        assert getattr(lib, name)(*dict(args, **over).values()) == 1, over
    if "ws" in args:
        assert getattr(lib, name)(*dict(args, ws_bytes=16).values()) == 2
    # nothing to do: no pointer is looked at
    assert getattr(lib, name)(*{k: None if isinstance(v, ctypes.c_void_p) else v for k, v in dict(args, R=0).items()}
                              .values()) == 0


def test_workspace_sizes(dsde):
    lib = dsde.load()
    for ws in (lib.dsde_sample_workspace_bytes, lib.dsde_distill_workspace_bytes):
        for bad in ((-1, 10), (1, 0), (1, 4194305), (1 << 31, 8), ((1 << 31) - 1, 9000)):
            assert ws(*bad) == 0, bad
        for V in (1, 8, 8192, 8193, 128256, 4194304):  # grows with both arguments
            sizes = [ws(R, V) for R in (0, 1, 7, 1000, 6000, 100000)]
            assert sizes == sorted(sizes) and sizes[1] > 0
        for R in (1, 300, 100000):
            sizes = [ws(R, V) for V in (1, 8192, 8193, 128256, 152064, 4194304)]
            assert sizes == sorted(sizes)
    assert lib.dsde_sample_workspace_bytes(1 << 30, 1) <= (192 << 20) + 1024


def calls(dsde, stream=None, **over):
    """Every call on CPU tensors, as name -> function."""
    i32 = dict(dtype=torch.int32)
    N, V, K = 3, 64, 4
    a = dict(z=torch.zeros(N, V, dtype=torch.bfloat16), T=torch.ones(N), u=torch.zeros(N), k=torch.zeros(N, **i32),
             p=torch.ones(N), m=torch.zeros(N), ids=torch.zeros(N, K, **i32), t=torch.zeros(N, K), lse=torch.zeros(N),
             w=torch.ones(N), record=torch.zeros(N, 32, dtype=torch.uint8), grad=None)
    a.update(over)
    return {
        "sample": lambda: dsde.sample(a["z"], a["T"], a["u"], top_k=a["k"], top_p=a["p"], min_p=a["m"], kept=True,
                                      stream=stream),
        "top_logits": lambda: dsde.top_logits(a["z"], 4, stream=stream),
        "distill_loss": lambda: dsde.distill_loss(a["z"], a["ids"], a["t"], teacher_lse=a["lse"], stream=stream),
        "distill_grad": lambda: dsde.distill_grad(a["z"], a["ids"], a["t"], a["record"], a["w"], grad=a["grad"],
                                                  stream=stream),
        "distill_step": lambda: dsde.distill_step(a["z"], a["ids"], a["t"], a["w"], teacher_lse=a["lse"],
                                                  grad=a["grad"], stream=stream),
    }


@pytest.mark.parametrize("name", ["sample", "top_logits", "distill_loss", "distill_grad", "distill_step"])
def test_logits_are_refused(dsde, name):
    z = torch.zeros(3, 64, dtype=torch.bfloat16)
    for bad, text in ((z, "logits must be a GPU tensor"), (z.half(), "bfloat16 or float32"),
                      (z.double(), "bfloat16 or float32"), (z[0], "rows, vocabulary|few dimensions"),
                      (z.view(3, 8, 8), "rows, vocabulary"), ([1.0], "rows, vocabulary|GPU tensor")):
        with pytest.raises(dsde.DsdeError, match=text):
            calls(dsde, z=bad)[name]()


def test_k_is_refused(dsde):
    z = torch.zeros(3, 64, dtype=torch.bfloat16)
    for k in (0, -1, 257):
        with pytest.raises(dsde.DsdeError, match="k must be in 1..256"):
            dsde.top_logits(z, k)


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

    monkeypatch.setattr(dsde, "_native", FakeNative())
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "Stream", FakeStream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
    monkeypatch.setattr(dsde, "new_sample_workspace", lambda R, V, device: torch.empty(8))
    monkeypatch.setattr(dsde, "new_distill_workspace", lambda N, V, device: torch.empty(8))
    want = "current" if stream is None else 78 if isinstance(stream, RawStream) else stream
    made = dict(sample=3, top_logits=5, distill_loss=4, distill_grad=1, distill_step=4)
    for name, f in calls(dsde, stream=stream).items():
        with Recorder(stack) as seen:
            f()
        assert seen.seen == [want] * made[name], name
