"""The cache's calls refuse tensors that require a gradient while gradients are recorded (they have no backward); the check
comes before the ones that need a GPU."""
import pytest
import torch

from test_kv_host import calls, dsde  # noqa: F401 (dsde is a fixture)

ASKS = "requires a gradient, which the cache's calls do not give"
GPU = "must be a GPU tensor"


def over(name):
    bf16 = dict(dtype=torch.bfloat16)
    return {name: torch.zeros(5, 4 if name == "q" else 2, 64, requires_grad=True, **bf16)}


@pytest.mark.parametrize("call,name", [("kv_write", "k"), ("kv_write", "v"), ("kv_attention", "q")])
def test_rows_that_want_a_gradient(dsde, call, name):  # noqa: F811
    if name == "v":  # behind k, which has to be a GPU tensor
        with torch.no_grad(), pytest.raises(dsde.DsdeError, match=GPU):
            calls(dsde, **over(name))[call]()
        return
    with pytest.raises(dsde.DsdeError, match=f"^{name} {ASKS}"):
        calls(dsde, **over(name))[call]()
    for quiet in (torch.no_grad, torch.inference_mode):
        with quiet(), pytest.raises(dsde.DsdeError, match=GPU):
            calls(dsde, **over(name))[call]()
    with pytest.raises(dsde.DsdeError, match=GPU):
        calls(dsde, **{name: over(name)[name].detach()})[call]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["q", "k", "v", "k_cache", "v_cache", "k_scale", "v_scale"])
def test_every_tensor(gpu_lib, name):
    """On the GPU, each of the calls' tensors: refused, and nothing is written; without recording, computed as ever."""
    i32 = dict(dtype=torch.int32, device="cuda")
    e4m3 = "scale" in name
    kc, vc = gpu_lib.new_kv_cache(4, 16, 2, 64, dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    for c in (kc, vc):
        c.view(torch.uint8).zero_()
    rows = torch.ones(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    a = dict(q=rows.clone(), k=rows[:, :2].clone(), v=rows[:, 2:].clone(), k_cache=kc, v_cache=vc,
             k_scale=torch.ones(2, device="cuda") if e4m3 else None, v_scale=torch.ones(2, device="cuda") if e4m3 else None)
    cache = lambda: (a["k_cache"], a["v_cache"])  # noqa: E731
    scales = lambda: dict(k_scale=a["k_scale"], v_scale=a["v_scale"])  # noqa: E731
    write = lambda: gpu_lib.kv_write(a["k"], a["v"], torch.arange(5, **i32), *cache(), **scales())  # noqa: E731
    attend = lambda: gpu_lib.kv_attention(a["q"], *cache(), torch.zeros(1, 4, **i32), torch.tensor([5], **i32),  # noqa: E731
                                          torch.tensor([0, 5], **i32), 5, **scales())["out"]
    want = attend()
    t = a[name]
    a[name] = t.clone().requires_grad_() if t.dtype != torch.float8_e4m3fn else t
    for call, uses in ((write, name != "q"), (attend, name not in ("k", "v"))):
        if uses:
            with pytest.raises(gpu_lib.DsdeError, match=f"^{name} {ASKS}"):
                call()
    with torch.no_grad():
        assert torch.equal(attend(), want)
        assert not write().any()
