"""The paged calls from their definitions: plan and write one token at a time on the host, attention in 64 bits,
with the error that each output may have."""
from __future__ import annotations

import math

import torch

EPS32 = 2.0 ** -24  # half a step of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: EPS32}


def blocks(tokens, page):
    return -(-tokens // page)


def plan(cached, fresh, free_pages, n_free, table, page, pages, T):
    """Lists in, lists out: (table, cu_q, kv_len, slots, pos, pages left, balance)."""
    table, n_free = [list(x) for x in table], min(max(n_free, 0), pages)
    width, rows, upto, left, balance = len(table[0]), 0, 0, n_free, n_free
    cu, kv_len, slots, pos = [0], [], [-1] * T, [-1] * T
    for r, (c, f) in enumerate(zip(cached, fresh)):
        first, rows = rows, rows + max(f, 0)
        cu.append(min(rows, T))
        ok = c >= 0 and f >= 0 and blocks(c + f, page) <= width and rows <= T
        need = blocks(c + f, page) - blocks(c, page) if ok else 0
        upto += need
        if not ok or (need > 0 and upto > n_free):
            kv_len.append(0)
            continue
        balance = n_free - upto
        for i in range(need):
            left -= 1
            table[r][blocks(c, page) + i] = free_pages[left]
        kv_len.append(c + f)
        for i in range(f):
            p = c + i
            page_id = table[r][p // page]
            pos[first + i] = p
            slots[first + i] = page_id * page + p % page if 0 <= page_id < pages else -1
    return table, cu, kv_len, slots, pos, left, balance


def attend(q, kp, vp, table, cu_q, kv_len, page, scale=0.0, p_half=None):
    """o, lse in 64 bits of the rows of cu_q (q [T, Hq, D], the pages as the library lays them out), and the largest
    error that o and lse may have. Rows of no request are NaN in all four.

    A logit x = scale q.k is a sum of D products in fp32 (and a product with the scale): off by at most
    (D + 2) 2^-24 scale |q|.|k|, dx. The running maximum cancels; exp2 of a fused product is within 2 ulp and
    its argument rounds once more: a weight is off by (dx + 2^-24 |x - max| + 2^-22) of itself, and by the half step
    p_half that it is rounded by before its product. The sums of the weights and of their products with V round once a key
    or less. Each division, rescaling (its factor rounds too, by at most 64 of them a row) and the joining
    of parts rounds once more, the last store by half a step of the type."""
    T, Hq, D = q.shape
    Hkv = kp.shape[1]
    G, dev, dt = Hq // Hkv, q.device, q.dtype
    scale = scale or 1.0 / math.sqrt(D)
    p_half = HALF[dt] if p_half is None else p_half
    new = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=dev)  # noqa: E731
    o, lse, o_tol, lse_tol = new(T, Hq, D), new(T, Hq), new(T, Hq, D), new(T, Hq)
    for r, total in enumerate(kv_len):
        a, b = cu_q[r], cu_q[r + 1]
        n = b - a
        if n <= 0:
            continue
        keys = torch.arange(total, device=dev)
        ids = torch.tensor([table[r][x] for x in range(blocks(total, page))], dtype=torch.long, device=dev)
        at = total - n + torch.arange(n, device=dev)  # positions
        late = keys[None] > at[:, None]
        empty = (at < 0)[:, None]
        for g in range(Hkv):
            k = kp[ids, g].reshape(-1, D)[:total].double()
            v = vp[ids, g].reshape(-1, D)[:total].double()
            for h in range(g * G, g * G + G):
                if total == 0:
                    o[a:b, h], lse[a:b, h], o_tol[a:b, h], lse_tol[a:b, h] = 0, -math.inf, 0, 0
                    continue
                x = q[a:b, h].double()
                # a row's sum runs over the keys that it sees: what is behind them may be anything
                s = torch.where(late, -math.inf, x @ k.T * scale)
                top = s.amax(1, keepdim=True).nan_to_num(nan=math.nan, neginf=0.0)
                w = (s - top).exp()
                l = w.sum(1, keepdim=True)
                w = w / torch.where(l > 0, l, 1.0)
                dx = torch.where(late, 0.0, (D + 2) * EPS32 * scale * (x.abs() @ k.abs().T))
                off = dx + EPS32 * torch.where(late, 0.0, (s - top).abs()) + 4 * EPS32
                sums = (total + 256) * EPS32
                dl = (w * off).sum(1, keepdim=True) + sums
                if bool(torch.isfinite(v).all()):
                    y, dy = w @ v, (w * (off + p_half)) @ v.abs() + (dl + sums) * (w @ v.abs())
                else:  # 0 times what is masked is no NaN here
                    y, dy = new(n, D), new(n, D)
                    for i in range(n):
                        m = int(at[i]) + 1
                        if m > 0:
                            y[i] = w[i, :m] @ v[:m]
                            dy[i] = (w[i, :m] * (off[i, :m] + p_half)) @ v[:m].abs() + (dl[i] + sums) * (w[i, :m] @ v[:m].abs())
                o[a:b, h] = torch.where(empty, 0.0, y)
                o_tol[a:b, h] = torch.where(empty, 0.0, dy * (1 + HALF[dt]) + HALF[dt] * y.abs() + 1e-30)
                z = (top + l.log())[:, 0]
                lse[a:b, h] = torch.where(empty[:, 0], -math.inf, z)
                lse_tol[a:b, h] = torch.where(empty[:, 0], 0.0, 2 * dl[:, 0] + dx.amax(1) + 8 * EPS32 * (z.abs() + top[:, 0].abs() + 1))
    return o, lse, o_tol, lse_tol


def check(name, got, ref, tol):
    """Every element within tol of ref; infinities and NaN where ref has them. Elements that are NaN in tol are not
    looked at, unless ref says infinity."""
    g, r = got.double(), ref
    assert g.shape == r.shape, (name, g.shape, r.shape)
    odd = ~torch.isfinite(r)
    same = (g == r) | (torch.isnan(g) & torch.isnan(r))
    assert bool(same[odd].all()), f"{name}: infinities or NaN in other places"
    d = (g - r).abs()[~odd]
    t = tol.expand_as(r)[~odd]
    assert bool(torch.isfinite(g[~odd]).all()), f"{name}: not finite"
    worst = float((d / t.clamp(min=1e-300)).max()) if d.numel() else 0.0
    print(f"  {name}: worst error over its bound {worst:.3f}, largest error {float(d.max()) if d.numel() else 0.0:.2e}", flush=True)
    assert bool((d <= t).all()), f"{name}: {int((d > t).sum())} of {d.numel()} outside, worst {worst:.2f} of the bound"
