"""The paged cache's operators in 64 bits (or integers), from their definitions."""
import math

import torch


def pages_of(lengths, page, P, seed=0):
    """Page lists of sequences of the given lengths, from a shuffled cache of P pages."""
    ids = torch.randperm(P, generator=torch.Generator().manual_seed(seed)).tolist()
    out = []
    for n in lengths:
        k = -(-n // page)
        out.append(ids[:k])
        ids = ids[k:]
    return out


def table_of(pages, width):
    t = torch.full((len(pages), width), -1, dtype=torch.int32)
    for i, x in enumerate(pages):
        t[i, :len(x)] = torch.tensor(x, dtype=torch.int32)
    return t


def prefix(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def attend(q, k, v, table, context, cu, scale, window=0, k_scale=None, v_scale=None, eps=2.0 ** -24):
    """out, lse and bounds of their errors: q [T, heads, D], k and v [P, key heads, page, D].

    ``eps`` is the rounding of a weight and of the result (half a step of their type).  A score is a sum of
    D products in 32 bits, off by (D + 4) 2^-23 of the sum of their sizes at most (accumulation, scale, reference);
    a weight is off by that and the exponential's 2^-21.  Of N tokens' weighted values at most N / 8 + 64 are added in a
    row.  With A = sum p |v|, out is off by (2 w + sum) A + eps (A + |out|)."""
    T, Hq, D = q.shape
    H, S = k.shape[1:3]
    G = Hq // H
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(context)):
        n, c = cu[b + 1] - cu[b], context[b]
        if n == 0 or c == 0:
            continue
        ids = table[b, :-(-c // S)].long()
        kk = k[ids].double().permute(1, 0, 2, 3).reshape(H, -1, D)[:, :c]
        vv = v[ids].double().permute(1, 0, 2, 3).reshape(H, -1, D)[:, :c]
        if k_scale is not None:
            kk, vv = kk * k_scale.double()[:, None, None], vv * v_scale.double()[:, None, None]
        for j in range(n):
            p = c - n + j
            lo = max(0, p - window + 1) if window else 0
            if p < 0:
                continue
            for h in range(Hq):
                key, val, x = kk[h // G, lo:p + 1], vv[h // G, lo:p + 1], q[cu[b] + j, h].double()
                z = scale * (key * x).sum(1)
                size = abs(scale) * (key * x).abs().sum(1)
                t = cu[b] + j
                if not torch.isfinite(z).any() and not torch.isnan(z).any() and (z < 0).all():
                    continue  # nothing but -inf
                lse[t, h] = torch.logsumexp(z, 0)
                w = torch.exp(z - lse[t, h])
                # a weight of 0 takes no part
                out[t, h] = (w[:, None] * val)[w != 0].sum(0)
                A = (w[:, None] * val.abs())[w != 0].sum(0)
                size = size[w > 1e-30].max() if (w > 1e-30).any() else size.max()
                ew = (D + 4) * 2.0 ** -23 * size + 2.0 ** -21
                es = (len(z) / 8 + 64) * 2.0 ** -24
                e_out[t, h] = (2 * ew + es) * A + eps * (A + out[t, h].abs())
                e_lse[t, h] = ew + es + 2.0 ** -22 * lse[t, h].abs() + 2.0 ** -22
    return out, lse, e_out, e_lse


def kv_map(sl, extra, kv_len, accepted, table, held, free, n_free, page, P, rows):
    """The state after the call and its outputs, as a loop over the sequences: lists of int."""
    B, W = len(sl), len(table[0])
    LAYOUT, STATE, PAGES = 1, 64, 256
    table, held, stack = [list(x) for x in table], list(held), list(free)
    n = [max(0, s + extra) for s in sl]
    base = [k + a + 1 for k, a in zip(kv_len, accepted)]
    cu, err, need = prefix(n), [0] * B, [None] * B
    for b in range(B):
        if sl[b] + extra < 0 or kv_len[b] < 0 or accepted[b] < -1:
            err[b] |= LAYOUT
        if not 0 <= held[b] <= W:
            err[b] |= STATE
        if not err[b]:
            need[b] = -(-(base[b] + n[b]) // page)
            if need[b] > W:
                err[b] |= PAGES
        if cu[b + 1] > rows:
            err[b] |= LAYOUT
        if kv_len[b] < 0 or accepted[b] < -1:
            base[b] = kv_len[b]
    back = [held[b] - need[b] if not err[b] and need[b] < held[b] else 0 for b in range(B)]
    take = [need[b] - held[b] if not err[b] and need[b] > held[b] else 0 for b in range(B)]
    top = n_free
    if not (0 <= n_free <= P and sum(back) <= P - n_free):
        for b in range(B):
            if back[b] or take[b]:
                err[b] |= STATE
        back = take = [0] * B
    for b in reversed(range(B)):
        for _ in range(back[b]):
            held[b] -= 1
            stack[top] = table[b][held[b]]
            table[b][held[b]] = -1
            top += 1
    out_of = top  # pages asked for so far may exceed what there is
    for b in range(B):
        if take[b]:
            out_of -= take[b]
            if out_of < 0:
                err[b] |= PAGES
                continue
            for _ in range(take[b]):
                top -= 1
                table[b][held[b]] = stack[top]
                held[b] += 1
    context = [0 if err[b] else base[b] + n[b] for b in range(B)]
    slots, pos = [-1] * rows, [-1] * rows
    for b in range(B):
        if err[b]:
            continue
        for j in range(n[b]):
            p = base[b] + j
            pos[cu[b] + j] = p
            pg = table[b][p // page]
            if 0 <= pg < P:
                slots[cu[b] + j] = pg * page + p % page
            else:
                err[b] = PAGES
    state = dict(table=table, held=held, free=stack, n_free=[top])
    return state, dict(base=base, context=context, cu_rows=cu, slots=slots, positions=pos, seq_err=err)
