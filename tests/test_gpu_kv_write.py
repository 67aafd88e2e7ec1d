"""dsde_kv_write: rows into their slots, bit for bit; e4m3 against the nearest of all its values."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


def cache(P, H, S, D, dtype, by_token, fill=3):
    """Keys and values whose every byte is `fill`."""
    n = torch.empty(0, dtype=dtype).element_size()
    out = []
    for _ in range(2):
        x = torch.full((P, S, H, D * n) if by_token else (P, H, S, D * n), fill, dtype=torch.uint8, device="cuda").view(dtype)
        out.append(x.transpose(1, 2) if by_token else x)
    return out


def bits(x):
    return x.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,H,D,S,by_token", [(1, 1, 16, 16, False), (5, 3, 48, 16, True), (1400, 8, 128, 16, False),
                                              (301, 5, 80, 32, False), (1000, 2, 256, 128, True), (77, 12, 64, 1024, False),
                                              (9, 40, 192, 16, True)])
def test_rows_land_in_their_slots(gpu_lib, T, H, D, S, by_token, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    P = -(-T // S) + 3
    both = torch.randn((T, 3 * H + 1, D), generator=g, device="cuda").to(DT[dtype])
    k, v = both[:, H:2 * H], both[:, 2 * H:3 * H]
    both[0, H, :3] = torch.tensor([float("nan"), float("inf"), -0.0])
    slots = torch.randperm(P * S, generator=g, device="cuda")[:T].int()
    slots[::7] = -1
    kc, vc = cache(P, H, S, D, DT[dtype], by_token)
    want = []
    for x, c in ((k, kc), (v, vc)):
        w = bits(c).clone()
        live = slots >= 0
        at = slots[live].long()
        w[at // S, :, at % S] = bits(x[live].contiguous())
        want.append(w)
    err = gpu_lib.kv_write(k, v, slots, kc, vc)
    assert torch.equal(bits(kc), want[0]) and torch.equal(bits(vc), want[1])
    assert not err.any()


def test_e4m3_is_the_nearest_value(gpu_lib):
    """Every bf16 number, and quotients near ties, against all 256 values; ties to the even one."""
    dev = "cuda"
    x = torch.arange(65536, dtype=torch.int32, device=dev).to(torch.int16).view(torch.bfloat16)
    k = torch.cat([x, x.flip(0)]).view(-1, 2, 64)
    T = k.shape[0]
    scale = torch.tensor([1.0, 0.37], device=dev)
    kc, vc = cache(T // 16, 2, 16, 64, DT["e4m3"], False, fill=0)
    slots = torch.arange(T, dtype=torch.int32, device=dev)
    gpu_lib.kv_write(k, k, slots, kc, vc, k_scale=scale, v_scale=scale)
    assert torch.equal(bits(kc), bits(vc))
    codes = torch.arange(127, dtype=torch.uint8, device=dev)  # 0 .. 448, ascending
    values = codes.view(DT["e4m3"]).double()
    y = (k.float() / scale[:, None]).double()  # the quotient in fp32, as documented
    got = bits(kc).permute(0, 2, 1, 3).reshape(T, 2, 64)
    nan = torch.isnan(y)
    assert torch.equal((got & 0x7f) == 0x7f, nan)
    a = y.abs().clamp(max=448.0).nan_to_num(0.0)
    up = torch.searchsorted(values, a).clamp(max=126)
    down = (up - 1).clamp(min=0)
    du, dd = values[up] - a, a - values[down]
    pick = torch.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, down)
    ok = ((got & 0x7f) == pick.to(torch.uint8)) & ((got >= 0x80) == torch.signbit(y))
    assert bool((ok | nan).all())


def test_e4m3_rows_and_layouts(gpu_lib):
    for T, H, D, S, by_token in ((700, 8, 128, 16, False), (33, 3, 80, 32, True), (5, 1, 16, 16, False), (90, 2, 256, 64, True)):
        g = torch.Generator(device="cuda").manual_seed(T)
        k, v = (torch.randn((T, H, D), generator=g, device="cuda").bfloat16() for _ in range(2))
        ks, vs = (0.01 + 0.05 * torch.rand(H, generator=g, device="cuda") for _ in range(2))
        P = -(-T // S) + 1
        slots = torch.randperm(P * S, generator=g, device="cuda")[:T].int()
        kc, vc = cache(P, H, S, D, DT["e4m3"], by_token)
        want = []
        for x, c, s in ((k, kc, ks), (v, vc, vs)):
            w = bits(c).clone()
            y = (x.float() / s[:, None]).clamp(-448, 448).to(DT["e4m3"])
            w[slots.long() // S, :, slots.long() % S] = bits(y)
            want.append(w)
        gpu_lib.kv_write(k, v, slots, kc, vc, k_scale=ks, v_scale=vs)
        assert torch.equal(bits(kc), want[0]) and torch.equal(bits(vc), want[1]), (T, H, D)


@pytest.mark.parametrize("dtype,T", [("bf16", 9000), ("e4m3", 17000)])
def test_more_rows_than_the_caches_hold(gpu_lib, dtype, T):
    H, D, S = 16, 128, 64
    g = torch.Generator(device="cuda").manual_seed(T)
    k, v = (torch.randn((T, H, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    scale = torch.full((H,), 0.25, device="cuda") if dtype == "e4m3" else None
    P = -(-T // S)
    slots = torch.randperm(P * S, generator=g, device="cuda")[:T].int()
    kc, vc = cache(P, H, S, D, DT[dtype], False)
    gpu_lib.kv_write(k, v, slots, kc, vc, k_scale=scale, v_scale=scale)
    for x, c in ((k, kc), (v, vc)):
        y = x if scale is None else (x.float() * 4.0).to(DT[dtype])  # a scale of a power of two
        assert torch.equal(bits(c)[slots.long() // S, :, slots.long() % S], bits(y))


def test_slots_out_of_range_are_flagged(gpu_lib):
    H, D, S, P = 2, 64, 16, 4
    buf = torch.full((P + 2, H, S, D), 7.0, device="cuda")  # the cache is its middle
    kc, vc = buf[1:P + 1], buf[1:P + 1].clone()
    k = torch.randn(6, H, D, device="cuda")
    slots = torch.tensor([0, -1, -2, P * S, 2 ** 31 - 1, P * S - 1], dtype=torch.int32, device="cuda")
    err = gpu_lib.kv_write(k, k, slots, kc, vc)
    assert err.tolist() == [0, 0, 256, 256, 256, 0]
    assert (buf[0] == 7).all() and (buf[-1] == 7).all() and torch.equal(kc, vc)
    assert torch.equal(kc[0, :, 0], k[0]) and torch.equal(kc[P - 1, :, S - 1], k[5])
    kc[0, :, 0] = 7
    kc[P - 1, :, S - 1] = 7
    assert (buf == 7).all()


def test_no_rows_and_versions(gpu_lib):
    kc, vc = gpu_lib.new_kv_cache(4, 16, 2, 64)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert gpu_lib.kv_write(none, none, torch.empty(0, dtype=torch.int32, device="cuda"), kc, vc).numel() == 0
    k = torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    before = kc._version
    gpu_lib.kv_write(k, k, torch.zeros(1, dtype=torch.int32, device="cuda"), kc, vc)
    assert kc._version > before and k._version == 0
