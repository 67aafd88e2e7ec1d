"""The paged key-value cache around a verification step, whose speed is followed: pages and
slots for the coming rows, writing those rows into the cache, and attention over it.

A case is a dict of plain values:

  op       map     dsde.kv_map: pages for a step's rows and the slot of each, and the same pages given back
           write   dsde.kv_write: a step's or a prompt's keys and values into their slots
           attend  dsde.kv_attention: a step's rows over each sequence's cache
  B        sequences
  lo, hi   tokens per sequence in the cache once the new rows are in it: spread evenly over their logarithm
  k        rows: 0: one row per sequence, k > 0: SL + 1 rows with SL = 1..k, evenly; -1: the whole prompt
  heads    key and value heads
  group    query heads per key head
  dim      elements per head
  page     tokens per page
  dtype    bf16 or fp32 queries, keys and values
  cache    bf16, fp32 or e4m3 (with a scale per head)
  window   (attend) how many tokens back a row sees, 0: all
  by_token (write, attend) the cache holds a token's heads side by side, and not a head's tokens
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp32": 4, "e4m3": 1}
SPARE = 64  # free pages beyond what a case needs


def _case(name, op, B, lo, hi, k, heads=8, group=4, dim=128, page=16, dtype="bf16", cache="", window=0, by_token=False):
    c = dict(op=op, B=B, lo=lo, hi=hi, k=k, heads=heads, group=group, dim=dim, page=page, dtype=dtype,
             cache=cache or dtype, window=window, by_token=by_token)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the look-ahead of the 64-sequence step: nothing but latency
        _case("map_b64", "map", 64, 100, 2000, 8),
        # one step of the controller loop's 1,024 sequences
        _case("map_b1024", "map", 1024, 64, 8192, 8),
        # a wave of new requests: pages for their prompts, given back when they end
        _case("map_prompts", "map", 256, 256, 8191, -1),
        # the rows of the 256-sequence step, cut out of a fused projection
        _case("write_b256", "write", 256, 300, 3000, 8),
        # prompts, into a cache that keeps a token's heads together
        _case("write_prompts", "write", 64, 200, 4001, -1, page=32, by_token=True),
        # prompts into a cache of 8 bits
        _case("write_e4m3", "write", 16, 129, 2048, -1, page=64, cache="e4m3"),
        # one user's next token after a short chat
        _case("attend_one", "attend", 1, 1000, 1000, 0),
        # one user's next token after a whole book: few rows, a long cache
        _case("attend_long", "attend", 1, 131072, 131072, 0, group=8),
        # a small draft model in fp32, a head of its own for each query head, short odd lengths
        _case("attend_b64_fp32", "attend", 64, 1, 2047, 0, heads=12, group=1, dim=64, dtype="fp32"),
        # the SL + 1 rows of every sequence of the 256-sequence step
        _case("attend_b256", "attend", 256, 256, 8192, 8),
        # one draft token for each of the loop's 1,024 sequences over a cache of 8 bits
        _case("attend_b1024", "attend", 1024, 64, 4096, 0, group=8, page=32, cache="e4m3"),
        # a model that looks back over a window, an odd head size, tokens' heads together
        _case("attend_window", "attend", 96, 500, 12000, 4, heads=4, group=6, dim=96, page=64, window=1024, by_token=True),
    ]


def draw(rng):
    op = rng.choice(["map", "write", "attend", "attend", "attend"])
    B = round(math.exp(rng.uniform(0, math.log(1024))))
    hi = round(math.exp(rng.uniform(math.log(64), math.log(131072 if op == "attend" else 8192))))
    lo = max(1, round(hi / math.exp(rng.uniform(0, math.log(64)))))
    page = rng.choice([16, 16, 32, 64, 128])
    heads = rng.choice([1, 2, 4, 8, 8, 12, 16])
    group = rng.choice([1, 2, 4, 5, 8, 8, 16])
    dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    cache = "e4m3" if dtype == "bf16" and rng.random() < 0.3 else dtype
    by_token = rng.random() < 0.3
    k = rng.choice({"map": [0, 1, 4, 8, 8, 16, -1], "write": [0, 4, 8, -1], "attend": [0, 0, 0, 1, 4, 8, 8, 16]}[op])
    window = rng.choice([0, 0, 0, 127, 1024]) if op == "attend" else 0
    if op == "map":
        heads, group, dim, dtype, cache, by_token = 8, 4, 128, "bf16", "bf16", False
    most = [_cost(c) for c in listed() if c["op"] == op]
    while True:
        c = _case(None, op, B, min(lo, hi), hi, k, heads, group, dim, page, dtype, cache, window, by_token)
        if all(x <= max(m[i] for m in most) for i, x in enumerate(_cost(c))):
            return c
        if B > 1 and (B > 64 or hi < 8192):
            B = (B + 1) // 2
        else:
            hi = (hi + 1) // 2


def _cost(case):
    """What a case takes of memory, its caches among it, and of arithmetic."""
    w = work(case)
    tokens = sum(_lengths(case)[0])
    cache = 0 if case["op"] == "map" else 2 * tokens * case["heads"] * case["dim"] * SIZE[case["cache"]]
    return w["bytes"], w["flops"], cache + 4 * tokens


def _lengths(case):
    """(tokens in the cache with the new rows, new rows) of every sequence."""
    B, lo, hi, k = case["B"], case["lo"], case["hi"], case["k"]
    total = [round(lo * (hi / lo) ** ((i + 0.5) / B)) for i in range(B)]
    rows = [n if k < 0 else 1 if k == 0 else min(n, 2 + i * 7 % k) for i, n in enumerate(total)]
    return total, rows


def _shuffled(case, seed):
    total, rows = _lengths(case)
    order = list(range(case["B"]))
    random.Random(seed).shuffle(order)
    return [total[i] for i in order], [rows[i] for i in order]


def _pages(case, total, r):
    """Pages in random order, as after a long run, in each sequence's order."""
    counts = [-(-n // case["page"]) for n in total]
    P = sum(counts) + SPARE
    ids = list(range(P))
    r.shuffle(ids)
    at, rows = 0, []
    for n in counts:
        rows.append(ids[at:at + n])
        at += n
    return P, rows, ids[at:]


def _table(rows, width, dev):
    t = np.full((len(rows), width), -1, dtype=np.int32)
    for i, x in enumerate(rows):
        t[i, :len(x)] = x
    return torch.from_numpy(t).to(dev)


def _ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _map_inputs(case, seed):
    """The pool as the last step left it: pages for each sequence's tokens so far."""
    total, n = _shuffled(case, seed)
    r = random.Random(seed + 1)
    prompt = case["k"] < 0
    extra = 0 if prompt else 1
    kept = [t - x for t, x in zip(total, n)]  # tokens that stay in the cache
    # the rows of the last step that were accepted are not in kv_len yet
    accepted = [-1 if prompt or a == 0 else r.randrange(min(4, a)) for a in kept]
    P, rows, free = _pages(case, total, r)
    held = [-(-a // case["page"]) for a in kept]
    free += [p for x, h in zip(rows, held) for p in x[h:]]
    r.shuffle(free)
    return dict(kv_len=[a - (c + 1) for a, c in zip(kept, accepted)], accepted=accepted, sl=[x - extra for x in n],
                extra=extra, rows=sum(n), P=P, held=held, table=[x[:h] for x, h in zip(rows, held)], free=free,
                width=-(-max(total) // case["page"]) + 1)


def _cu(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _cache(case, P, fill, g, dev):
    """Keys and values [pages, heads, page, dim] of the case's layout, and their scales."""
    H, S, D = case["heads"], case["page"], case["dim"]
    shape = (P, S, H, D) if case["by_token"] else (P, H, S, D)
    out = []
    for strength in (1.0, 0.5):
        x = torch.zeros(shape, dtype=DT[case["cache"]], device=dev)
        step = max(1, (1 << 27) // x[0].numel())
        if fill:
            # heads differ in strength, and a few channels stand out
            s = 0.5 + torch.rand((1, 1, H, 1) if case["by_token"] else (1, H, 1, 1), generator=g, device=dev)
            c = 1.0 + 4.0 * (torch.rand(D, generator=g, device=dev) > 0.97)
            for i in range(0, P, step):
                y = torch.randn((min(step, P - i),) + shape[1:], generator=g, device=dev)
                x[i:i + step] = (y * s * c * strength).to(x.dtype)
        out.append(x.transpose(1, 2) if case["by_token"] else x)
    scale = [0.01 + 0.05 * torch.rand(H, generator=g, device=dev) if case["cache"] == "e4m3" else None for _ in range(2)]
    return out, scale


def _write_inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(1_000_003 * seed + 31)
    total, n = _shuffled(case, seed)
    P, pages, _ = _pages(case, total, random.Random(seed + 1))
    T, H, D, S = sum(n), case["heads"], case["dim"], case["page"]
    slots = np.concatenate([np.asarray(x, dtype=np.int64)[np.arange(t - m, t) // S] * S + np.arange(t - m, t) % S
                            for x, t, m in zip(pages, total, n)])
    # queries, keys and values of a row lie together, as a fused projection leaves them
    Q = H * case["group"]
    both = torch.empty((T, Q + 2 * H, D), dtype=DT[case["dtype"]], device=dev)
    for i in range(0, T, 8192):
        both[i:i + 8192] = torch.randn((min(8192, T - i), Q + 2 * H, D), generator=g, device=dev).to(both.dtype)
    (kc, vc), (ks, vs) = _cache(case, P, False, g, dev)
    return dict(k=both[:, Q:Q + H], v=both[:, Q + H:], slots=torch.from_numpy(slots).int().to(dev), k_cache=kc, v_cache=vc,
                k_scale=ks, v_scale=vs)


def _attend_inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(1_000_003 * seed + 37)
    total, n = _shuffled(case, seed)
    P, pages, _ = _pages(case, total, random.Random(seed + 1))
    H, D = case["heads"], case["dim"]
    (kc, vc), (ks, vs) = _cache(case, P, True, g, dev)
    if ks is not None:  # keys and values of ordinary size after their scales
        ks, vs = 0.5 + ks, 0.5 + vs
    q = torch.randn((sum(n), H * case["group"], D), generator=g, device=dev)
    q = q * (0.3 + 1.2 * torch.rand((1, H * case["group"], 1), generator=g, device=dev))
    return dict(q=q.to(DT[case["dtype"]]), k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs,
                table=_table(pages, -(-case["hi"] // case["page"]), dev), context=_ints(total, dev), cu_rows=_ints(_cu(n), dev),
                max_rows=max(1, case["k"] + 1))


def prepare(case, seed):
    dev = torch.device("cuda")
    if case["op"] == "map":
        x = _map_inputs(case, seed)
        B, P = case["B"], x["P"]
        free = torch.full((P,), -1, dtype=torch.int32)
        free[:len(x["free"])] = torch.tensor(x["free"], dtype=torch.int32)
        s = dict(sl=_ints(x["sl"], dev), kv_len=_ints(x["kv_len"], dev), accepted=_ints(x["accepted"], dev), extra=x["extra"],
                 rows=x["rows"], page=case["page"], none=torch.zeros(B, dtype=torch.int32, device=dev),
                 pool=dict(table=_table(x["table"], x["width"], dev), held=_ints(x["held"], dev), free=free.to(dev),
                           n_free=_ints([len(x["free"])], dev)))
        if own:
            import paper_2509_01083_amd as dsde
            s["workspace"] = dsde.new_kv_map_workspace(B, dev)
            s["out"], s["back"] = dsde.new_kv_map_out(B, x["rows"], dev), dsde.new_kv_map_out(B, 0, dev)
    elif case["op"] == "write":
        s = _write_inputs(case, seed)
        if own:
            s["row_err"] = torch.empty(len(s["slots"]), dtype=torch.int32, device=dev)
    else:
        s = _attend_inputs(case, seed)
        s["window"] = case["window"]
        if own:
            import paper_2509_01083_amd as dsde
            s["workspace"] = dsde.new_kv_attention_workspace(case["B"], case["heads"], case["group"], s["max_rows"], case["dim"], dev)
            s["out"] = dict(out=torch.empty_like(s["q"]), lse=torch.empty(s["q"].shape[:2], device=dev),
                            seq_err=torch.empty(case["B"], dtype=torch.int32, device=dev))
    return dict(s, op=case["op"])


def _plain_map(pool, kv_len, accepted, sl, extra, page, rows):
    table, held, free, n_free = pool["table"], pool["held"], pool["free"], pool["n_free"]
    B, W = table.shape
    dev = table.device
    n = sl.long() + extra
    base = kv_len.long() + (0 if accepted is None else accepted.long() + 1)
    need = (base + n + page - 1) // page
    cu = torch.zeros(B + 1, dtype=torch.int64, device=dev)
    cu[1:] = n.cumsum(0)
    cols = torch.arange(W, device=dev)[None, :]
    P = free.shape[0]
    stack = torch.cat([free.long(), free.new_zeros(1).long()])
    # pages behind the need go back, the last sequence's last one first
    back = (cols >= need[:, None]) & (cols < held[:, None])
    rank = back.flatten().flip(0).cumsum(0).flip(0).view(B, W) - 1
    stack.scatter_(0, torch.where(back, n_free + rank, P).flatten(), table.long().flatten())
    count = n_free + back.sum()
    grow = (cols >= held[:, None]) & (cols < need[:, None])
    rank = grow.flatten().cumsum(0).view(B, W) - 1
    page_of = stack[torch.where(grow, count - 1 - rank, P)]
    new = torch.where(grow, page_of, torch.where(back, -1, table.long()))
    table.copy_(new)
    held.copy_(need)
    free.copy_(stack[:P])
    n_free.copy_(count - grow.sum())
    t = torch.arange(rows, device=dev)
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = base[b] + t - cu[b]
    slots = new[b, pos // page] * page + pos % page
    return dict(base=base.int(), context=(base + n).int(), cu_rows=cu.int(), slots=slots.int(), positions=pos.int())


def _plain_write(s):
    out = {}
    for name in ("k", "v"):
        x, cache, scale = s[name], s[name + "_cache"], s[name + "_scale"]
        S = cache.shape[2]
        if scale is not None:
            x = (x.float() / scale[:, None]).clamp(-448.0, 448.0).to(cache.dtype)
        slot = s["slots"].long()
        bits = cache.view(torch.uint8) if scale is not None else cache  # no indexed writes in 8 bits of float
        bits[slot // S, :, slot % S] = x.view(torch.uint8) if scale is not None else x
        out[name + "_cache"] = cache
    return out


def _values(s):
    """The caches of a write, those of 8 bits as the values they stand for."""
    if s["k_scale"] is None:
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    return {n + "_cache": s[n + "_cache"].float() * s[n + "_scale"][:, None, None] for n in ("k", "v")}


def _plain_attend(s):
    q, table, context, cu = s["q"].float(), s["table"].long(), s["context"].long(), s["cu_rows"].long()
    H, S, D = s["k_cache"].shape[1:]
    G, R, B = q.shape[1] // H, s["max_rows"], len(context)
    L = table.shape[1] * S
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=q.device)
    pos = torch.arange(L, device=q.device)
    some = max(1, (1 << 29) // (L * H * D))  # sequences at once
    for i in range(0, B, some):
        ids = table[i:i + some].clamp(min=0)
        c = len(ids)

        def rows(cache, scale):
            x = cache[ids.flatten()].float()
            x = x.view(c, -1, H, S, D).permute(0, 2, 1, 3, 4).reshape(c, H, L, D)
            return x if scale is None else x * scale[:, None, None]

        first, n = cu[i:i + c], cu[i + 1:i + c + 1] - cu[i:i + c]
        j = torch.arange(R, device=q.device)
        live = j < n[:, None]  # [c, R]
        at = (first[:, None] + j).clamp(max=len(q) - 1)
        y = q[at].view(c, R, H, G, D).permute(0, 2, 4, 1, 3).reshape(c, H, D, R * G)
        score = (rows(s["k_cache"], s["k_scale"]) @ y) * D ** -0.5  # [c, H, L, R G]
        here = (context[i:i + c] - n)[:, None] + j
        seen = pos[None, :, None] <= here[:, None, :]
        if s["window"]:
            seen &= pos[None, :, None] > here[:, None, :] - s["window"]
        seen = seen.repeat_interleave(G, dim=2)[:, None]
        score.masked_fill_(~seen, -math.inf)
        top = score.amax(2, keepdim=True).clamp(min=-1e30)
        p = (score - top).exp_()
        total = p.sum(2, keepdim=True)
        o = (p / total).transpose(2, 3).contiguous() @ rows(s["v_cache"], s["v_scale"])  # [c, H, R G, D]
        o = o.view(c, H, R, G, D).permute(0, 2, 1, 3, 4).reshape(c, R, H * G, D)
        z = (total.log() + top).view(c, H, R, G).permute(0, 2, 1, 3).reshape(c, R, H * G)
        where = torch.where(live, at, len(q)).flatten()  # the rows of shorter sequences end behind the last
        out = torch.cat([out, out[:1]]).index_copy_(0, where, o.flatten(0, 1))[:-1]
        lse = torch.cat([lse, lse[:1]]).index_copy_(0, where, z.flatten(0, 1))[:-1]
    return dict(out=out.to(s["q"].dtype), lse=lse)


def _plain(s):
    if s["op"] == "map":
        o = _plain_map(s["pool"], s["kv_len"], s["accepted"], s["sl"], s["extra"], s["page"], s["rows"])
        before = s["none"] if s["extra"] == 0 else s["kv_len"]
        back = None if s["extra"] == 0 else s["accepted"]
        _plain_map(s["pool"], before, back, s["none"], 0, s["page"], 0)
        return dict(o, **s["pool"])
    if s["op"] == "write":
        _plain_write(s)
        return _values(s)
    return _plain_attend(s)


def run(s):
    if not own:
        return _plain(s)
    import paper_2509_01083_amd as dsde
    if s["op"] == "map":
        # the coming step's rows, then, called off or ended, what is behind the tokens that stay
        o = dsde.kv_map(s["sl"], s["kv_len"], s["pool"], s["page"], s["rows"], extra=s["extra"], accepted=s["accepted"],
                        out=s["out"], workspace=s["workspace"])
        before = s["none"] if s["extra"] == 0 else s["kv_len"]
        back = None if s["extra"] == 0 else s["accepted"]
        dsde.kv_map(s["none"], before, s["pool"], s["page"], 0, extra=0, accepted=back, out=s["back"],
                    workspace=s["workspace"])
        return dict({k: o[k] for k in ("base", "context", "cu_rows", "slots", "positions")}, **s["pool"])
    if s["op"] == "write":
        dsde.kv_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                      row_err=s["row_err"])
        return _values(s)
    o = dsde.kv_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["context"], s["cu_rows"], s["max_rows"],
                          window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=True, out=s["out"],
                          workspace=s["workspace"])
    return dict(out=o["out"], lse=o["lse"])


def work(case):
    """The map: its arrays once and the pages that move, each way.  The write: each row in and out once.
    The attention: the keys and values that any of a sequence's rows sees once, its rows in and out."""
    total, n = _lengths(case)
    B, T, S, H, D = case["B"], sum(n), case["page"], case["heads"], case["dim"]
    if case["op"] == "map":
        moved = sum(-(-t // S) - -(-(t - x) // S) for t, x in zip(total, n))
        return {"bytes": 2 * 28 * B + 8 * T + 16 * moved, "flops": 0}
    e, c = SIZE[case["dtype"]], SIZE[case["cache"]]
    if case["op"] == "write":
        return {"bytes": 2 * T * H * D * (e + c) + 4 * T, "flops": 2 * T * H * D}
    seen = lambda t: min(t, case["window"]) if case["window"] else t  # noqa: E731
    keys = sum(min(t, seen(t) + x - 1) for t, x in zip(total, n))
    pairs = sum(seen(t - j) for t, x in zip(total, n) for j in range(x))
    return {"bytes": 2 * keys * H * D * c + T * H * case["group"] * (2 * D * e + 4), "flops": 4 * pairs * H * case["group"] * D}


def _exact_map(case, seed):
    x = _map_inputs(case, seed)
    S = case["page"]
    free, rows, n = list(x["free"]), [list(t) for t in x["table"]], [a + x["extra"] for a in x["sl"]]
    base = [a + c + 1 for a, c in zip(x["kv_len"], x["accepted"])]
    for t, b, m in zip(rows, base, n):
        while len(t) * S < b + m:
            t.append(free.pop())
    pos = [np.arange(b, b + m) for b, m in zip(base, n)]
    slots = [np.asarray(t, dtype=np.int64)[p // S] * S + p % S for t, p in zip(rows, pos)]
    stays = [0 if x["extra"] == 0 else b for b in base]
    for t, b in reversed(list(zip(rows, stays))):
        while len(t) > -(-b // S):
            free.append(t.pop())
    dev = torch.device("cuda")
    stack = np.full(x["P"], -1, dtype=np.int64)
    stack[:len(free)] = free
    i32 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(dev)  # noqa: E731
    return dict(base=i32(base), context=i32([b + m for b, m in zip(base, n)]), cu_rows=i32(_cu(n)),
                slots=i32(np.concatenate(slots)), positions=i32(np.concatenate(pos)), table=_table(rows, x["width"], dev),
                held=i32([len(t) for t in rows]), free=i32(stack), n_free=i32([len(free)]))


def _exact_write(case, seed):
    x = _write_inputs(case, seed)
    S = case["page"]
    out = {}
    for name in ("k", "v"):
        cache, scale = x[name + "_cache"], x[name + "_scale"]
        y = x[name].double()
        if scale is not None:
            y = (y / scale.double()[:, None]).clamp(-448, 448)
            # to the nearest of 8 steps in a power of two, and of 2^-9 below 2^-6; ties to even
            step = torch.exp2(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent.double() - 4)
            y = torch.round(y / step) * step * scale.double()[:, None]
        flat = torch.zeros(cache.shape[0] * S, cache.shape[1], cache.shape[3], dtype=torch.float64, device=y.device)
        flat[x["slots"].long()] = y
        out[name + "_cache"] = flat.view(cache.shape[0], S, cache.shape[1], cache.shape[3]).transpose(1, 2)
    return out


def _exact_attend(case, seed):
    x = _attend_inputs(case, seed)
    total, n = _shuffled(case, seed)
    H, S, D, G = case["heads"], case["page"], case["dim"], case["group"]
    q = x["q"].double()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    at = 0
    for b, (t, m) in enumerate(zip(total, n)):
        low = max(0, t - m + 1 - case["window"]) if case["window"] else 0
        first = low // S
        ids = x["table"][b, first:-(-t // S)].long()
        for h in range(H):
            k, v = (x[c][ids, h].double().reshape(-1, D)[low - first * S:t - first * S] for c in ("k_cache", "v_cache"))
            if x["k_scale"] is not None:
                k, v = k * x["k_scale"][h].double(), v * x["v_scale"][h].double()
            for j in range(m):
                end = t - m + 1 + j - low
                start = max(0, end - case["window"]) if case["window"] else 0
                rows = slice(h * G, h * G + G)
                z = q[at + j, rows] @ k[start:end].T.contiguous() / math.sqrt(D)
                lse[at + j, rows] = torch.logsumexp(z, dim=1)
                out[at + j, rows] = torch.softmax(z, dim=1) @ v[start:end]
        at += m
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] == "map":
        return _exact_map(case, seed)
    if case["op"] == "write":
        return _exact_write(case, seed)
    # a few launches for every sequence, head and row
    if case["B"] * case["heads"] * (case["k"] + 2) > 40000:
        return None
    return _exact_attend(case, seed)
