"""Serving over a paged K/V cache, as timed cases: the operators that a step of many requests runs.

A case is a plain dict. ``kind`` says which operator one pass goes through:

* ``plan``: block tables, slot maps and token positions of a step, from the requests' lengths;
* ``write``: the step's new K and V rows into their cache slots;
* ``attend``: attention of every request's new tokens (one of them: decoding) over its cached
  keys and values, causal inside the chunk.

The lengths of a case's requests are drawn from its own numbers (``_lengths``), so that the work of
a case is known without its inputs. ``run`` computes the operators in plain torch, or, where
``own`` is true, through this package's entry points; ``exact`` gives the same from the definition
in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _case(kind, R, new, cached, Hq=8, Hkv=8, D=128, page=64, dtype="bf16", ones=0.0, fused=False, spare=1.0, name=None):
    """new, cached: (least, most) new and cached tokens of a request, spread over the logarithm; ones: the share
    of requests that bring one token whatever `new` says; fused: q, k, v are slices of one projection's rows;
    spare: pages in the free list over those needed."""
    c = dict(kind=kind, R=R, new_lo=new[0], new_hi=new[1], cached_lo=cached[0], cached_hi=cached[1], Hq=Hq, Hkv=Hkv, D=D,
             page=page, dtype=dtype, ones=ones, fused=fused, spare=spare)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decoding step of 64 running requests: the smallest plan, bound by latency
        _case("plan", 64, (1, 1), (100, 32000), page=16, name="plan_decode_64"),
        # a step that takes in prompts for 256 requests while the pool runs short: the last ones have to wait
        _case("plan", 256, (64, 4096), (0, 8192), page=64, ones=0.25, spare=0.9, name="plan_prompts_256"),
        # one token of each of 64 requests into the cache
        _case("write", 64, (1, 1), (100, 4000), page=16, fused=True, name="write_decode_64"),
        # prompts of 24 requests into the cache
        _case("write", 24, (100, 4096), (0, 1000), page=64, name="write_prompts_24"),
        # the smallest attention call: one token of one request of a debugging-sized fp32 model
        _case("attend", 1, (1, 1), (777, 777), 2, 2, 64, 16, "fp32", name="decode_1_fp32"),
        # a decoding step of 64 requests of ragged lengths with grouped heads
        _case("attend", 64, (1, 1), (1000, 32000), 32, 8, 128, 16, fused=True, name="decode_64_gqa"),
        # one request at the end of a context of 256K tokens
        _case("attend", 1, (1, 1), (262143, 262143), 32, 8, 128, 64, fused=True, name="decode_1_256k"),
        # a few drafted tokens of each request to be verified in one pass, heads of 64
        _case("attend", 16, (2, 6), (1000, 24000), 12, 4, 64, 32, name="verify_16_d64"),
        # a chunk of a long prompt at the training length, 8 heads
        _case("attend", 1, (2048, 2048), (96256, 96256), 8, 8, 128, 64, fused=True, name="chunk_2k_96k"),
        # decoding requests and prompt chunks in one step
        _case("attend", 24, (100, 512), (500, 16000), 32, 8, 128, 32, ones=0.8, fused=True, name="mixed_24"),
        # two whole prompts without a cached token
        _case("attend", 2, (7000, 8192), (0, 0), 16, 16, 128, 64, name="prompt_8k"),
        # chunks of an fp32 model with grouped heads: numerics studies
        _case("attend", 3, (64, 256), (1000, 4000), 8, 2, 128, 16, "fp32", name="chunk_fp32_gqa"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1)))) - 1)) if hi > lo else lo


def _lengths(c):
    """(cached, new) tokens of every request."""
    rng = random.Random("%(R)d %(new_lo)d %(new_hi)d %(cached_lo)d %(cached_hi)d %(page)d" % c)
    new = [1 if rng.random() < c["ones"] else max(1, _log_int(rng, c["new_lo"], c["new_hi"])) for _ in range(c["R"])]
    return [_log_int(rng, c["cached_lo"], c["cached_hi"]) for _ in range(c["R"])], new


def _flops(c):
    cached, new = _lengths(c)
    return 4 * c["D"] * c["Hq"] * sum(n * a + n * (n + 1) // 2 for a, n in zip(cached, new))


def draw(rng):
    """One more case: 1 to 256 requests of up to 256K tokens, chunks of up to 8K tokens, every page size, type, head
    layout and kind."""
    while True:
        kind = rng.choice(["plan", "plan", "write", "write"] + ["attend"] * 8)
        R = _log_int(rng, 1, 256)
        page = rng.choice([16, 16, 32, 64, 64, 128, 256])
        mode = rng.choice(["decode", "decode", "verify", "chunk", "mixed", "prompt"])
        new = {"decode": (1, 1), "verify": (1, 8), "prompt": (16, 8192)}.get(mode, (16, _log_int(rng, 32, 4096)))
        cached = (0, 0) if mode == "prompt" else (rng.choice([0, 100, 1000]), _log_int(rng, 1000, 262144))
        Hkv = rng.choice([1, 2, 3, 4, 8, 8, 16])
        G = rng.choice([1, 1, 2, 3, 4, 4, 8])
        dtype = "fp32" if rng.random() < 0.2 else "bf16"
        c = _case(kind, R, new, cached, Hkv * G, Hkv, rng.choice([64, 128, 128]), page, dtype,
                  rng.choice([0.5, 0.9]) if mode == "mixed" else 0.0, rng.random() < 0.5,
                  rng.choice([1.0, 1.0, 1.3, 0.8]) if kind == "plan" else 1.0)
        old, fresh = _lengths(c)
        e = 4 if dtype == "fp32" else 2
        keys = R * (max(old) + max(fresh))
        if Hkv * G > 64 or sum(fresh) > (131072 if kind == "plan" else 32768):
            continue
        # no dearer than the largest listed cases, and the plain form's padded batch fits the card
        if kind == "attend" and (_flops(c) > (4e10 if dtype == "fp32" else 8e11) or sum(old) * Hkv * c["D"] * e > 3e9
                                 or keys * max(fresh) * c["Hq"] > 4e9 or keys * Hkv * c["D"] > 2e9):
            continue
        if kind == "write" and (sum(old) + sum(fresh)) * Hkv * c["D"] * e > 1e9 or kind == "plan" and sum(old) > 8 * 10 ** 6:
            continue
        return c


# ------------------------------------------------------------------ inputs

def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(4000 + seed)
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _blocks(tokens, page):
    return -(-tokens // page)


def prepare(case, seed):
    """What a serving program holds before the call: the step's rows, the pool of pages (a random order of them in the
    tables, as after some time of use), tables and lengths on the device, and the buffers it keeps for outputs."""
    c, g = case, _gen(seed)
    old, new = _lengths(c)
    R, T, Hq, Hkv, D, page, dt = c["R"], sum(new), c["Hq"], c["Hkv"], c["D"], c["page"], _dtype(c)
    after = [a + n for a, n in zip(old, new)]
    held = [_blocks(a, page) for a in (old if c["kind"] == "plan" else after)]
    wanted = sum(_blocks(a, page) for a in after)
    pages = max(wanted, sum(held)) + 8
    width = max(_blocks(a, page) for a in after)
    s = dict(c=c, T=T, width=width, pages=pages, most_new=max(new), most_keys=max(after), old=_ints(old), new=_ints(new),
             kv_len=_ints(after), cu_q=torch.cat([_ints([0]), _ints(new).cumsum(0).to(torch.int32)]))
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    counts = torch.tensor(held, device="cuda")
    first = counts.cumsum(0) - counts
    cols = torch.arange(width, device="cuda")
    at = (first[:, None] + cols).clamp(max=pages - 1)
    s["table"] = torch.where(cols < counts[:, None], order[at], torch.zeros_like(order[at])).contiguous()
    if c["kind"] == "plan":
        free = order[sum(held):]
        n = min(free.numel(), int((wanted - sum(held)) * c["spare"]))
        s["free"], s["n_free"] = torch.cat([free[:n], order[: pages - n]]).contiguous(), _ints([n])
        s.update(cu_out=_ints([0] * (R + 1)), len_out=_ints([0] * R), slots=_ints([0] * T), pos=_ints([0] * T), left=_ints([0]))
        return s
    f = dict(dtype=torch.float32, device="cuda", generator=g)
    if c["fused"]:
        rows = torch.randn(T, Hq + 2 * Hkv, D, **f).to(dt)
        s["q"], s["k"], s["v"] = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    else:
        s["q"], s["k"], s["v"] = (torch.randn(T, H, D, **f).to(dt) for H in (Hq, Hkv, Hkv))
    s["kp"], s["vp"] = (torch.empty(pages, Hkv, page, D, dtype=dt, device="cuda").normal_(generator=g) for _ in range(2))
    if c["kind"] == "write":
        t = torch.arange(T, device="cuda")
        r = torch.searchsorted(s["cu_q"][1:].contiguous(), t.to(torch.int32), right=True)
        p = s["old"].long()[r] + t - s["cu_q"].long()[r]
        s["slots"] = (s["table"].long()[r, p // page] * page + p % page).to(torch.int32)
        del s["q"]
    else:
        s["o"] = torch.empty(T, Hq, D, dtype=dt, device="cuda")
        s["lse"] = torch.empty(T, Hq, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    s = state
    if own:
        return _own(s)
    return {"plan": _plan, "write": _write, "attend": _attend}[s["c"]["kind"]](s)


def _own(s):
    import paper_2605_06554_amd as lh
    c = s["c"]
    if "step" not in s:  # the step's description and the workspace, which a program keeps beside its buffers
        s["step"] = lh.paged(c["R"], s["width"], s["T"], s["pages"], c["page"], c["Hq"], c["Hkv"], c["D"], _dtype(c))
        s["ws"] = lh.paged_workspace(s["step"]) if c["kind"] == "attend" else None
    pc = s["step"]
    if c["kind"] == "plan":
        lh.lh_page_plan(pc, s["old"], s["new"], s["free"], s["n_free"], s["table"], s["cu_out"], s["len_out"], s["slots"],
                        s["pos"], s["left"])
        return dict(table=s["table"], cu_q=s["cu_out"], kv_len=s["len_out"], slots=s["slots"], pos=s["pos"], n_left=s["left"])
    if c["kind"] == "write":
        lh.lh_page_write(pc, s["k"], s["v"], s["slots"], s["kp"], s["vp"])
        return dict(kp=s["kp"], vp=s["vp"])
    lh.lh_sdpa_paged(pc, s["q"], s["kp"], s["vp"], s["table"], s["cu_q"], s["kv_len"], s["o"], s["lse"], s["ws"])
    return dict(o=s["o"], lse=s["lse"])


def _plan(s):
    """Pages are handed out from the end of the free list in request order; from the first request for which they do
    not suffice, none that needs a page gets one (its length is 0, its slots are -1)."""
    page, T, dev = s["c"]["page"], s["T"], "cuda"
    old, new = s["old"].long(), s["new"].long()
    after = old + new
    cu = torch.nn.functional.pad(new.cumsum(0), (1, 0))
    own_, all_ = (old + page - 1) // page, (after + page - 1) // page
    need = all_ - own_
    upto = need.cumsum(0)
    n_free = s["n_free"].long()
    ok = (need == 0) | (upto <= n_free)
    t = torch.arange(T, device=dev)
    r = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    pos = old[r] + t - cu[r]
    block = pos // page
    rank = upto[r] - need[r] + block - own_[r]  # of the block among the step's new ones; below own_: an old one
    taken = s["free"][(n_free - 1 - rank).clamp(min=0)]
    ids = torch.where(block >= own_[r], taken, s["table"][r, block])
    table = s["table"].clone()
    table[r, block] = torch.where(ok[r], ids, table[r, block])
    slots = torch.where(ok[r], ids.long() * page + pos % page, -1)
    left = n_free - torch.where(ok, upto, 0).amax().clamp(min=0) if T else n_free
    i32 = torch.int32
    return dict(table=table, cu_q=cu.to(i32), kv_len=torch.where(ok, after, 0).to(i32), slots=slots.to(i32),
                pos=torch.where(ok[r], pos, -1).to(i32), n_left=left.to(i32))


def _write(s):
    page, slot = s["c"]["page"], s["slots"].long()
    s["kp"][slot // page, :, slot % page] = s["k"]
    s["vp"][slot // page, :, slot % page] = s["v"]
    return dict(kp=s["kp"], vp=s["vp"])


def _attend(s):
    """A padded batch: [R, heads, new tokens, keys]."""
    c = s["c"]
    R, Hq, Hkv, D, page, n, m = c["R"], c["Hq"], c["Hkv"], c["D"], c["page"], s["most_new"], s["most_keys"]
    G, dev = Hq // Hkv, "cuda"
    j, i = torch.arange(m, device=dev), torch.arange(n, device=dev)
    ids = s["table"].long()[:, j // page]  # [R, m]
    keys = s["kp"][ids, :, j % page].float().permute(0, 2, 3, 1).contiguous()  # [R, Hkv, D, m]
    values = s["vp"][ids, :, j % page].float().permute(0, 2, 1, 3).contiguous()  # [R, Hkv, m, D]
    cu, total = s["cu_q"].long(), s["kv_len"].long()
    rows = (cu[:-1, None] + i).clamp(max=s["T"] - 1)  # [R, n]
    q = s["q"][rows].float().view(R, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n, D)
    x = torch.matmul(q, keys).mul_(1.0 / math.sqrt(D)).view(R, Hkv, G, n, m)
    place = (total - (cu[1:] - cu[:-1]))[:, None] + i  # [R, n]
    x.masked_fill_((j > place[:, :, None])[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    norm = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(R, Hkv, G * n, m), values).view(R, Hkv, G, n, D) / norm
    lse = (top + norm.log())[..., 0]
    t = torch.arange(s["T"], device=dev)
    r = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    a = t - cu[r]
    return dict(o=o.permute(0, 3, 1, 2, 4)[r, a].reshape(s["T"], Hq, D).to(_dtype(c)),
                lse=lse.permute(0, 3, 1, 2)[r, a].reshape(s["T"], Hq).contiguous())


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    old, new = _lengths(c)
    T, page, e = sum(new), c["page"], 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "plan":
        taken = sum(_blocks(a + n, page) - _blocks(a, page) for a, n in zip(old, new))
        return {"bytes": 4 * (4 * c["R"] + 2 * T + 2 * taken + sum(a % page > 0 for a in old)), "flops": 0}
    row = c["Hkv"] * c["D"] * e
    if c["kind"] == "write":
        return {"bytes": 4 * T * row + 4 * T, "flops": 0}
    b = 2 * sum(a + n for a, n in zip(old, new)) * row + 2 * T * c["Hq"] * c["D"] * e + 4 * T * c["Hq"]
    return {"bytes": b + 4 * sum(_blocks(a + n, page) for a, n in zip(old, new)), "flops": _flops(c)}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(case, seed):
    c, s = case, prepare(case, seed)
    page = c["page"]
    if c["kind"] == "plan":
        return _exact_plan(c, s)
    if c["kind"] == "write":
        kp, vp = s["kp"].double(), s["vp"].double()
        for t, slot in enumerate(s["slots"].tolist()):
            kp[slot // page, :, slot % page] = s["k"][t].double()
            vp[slot // page, :, slot % page] = s["v"][t].double()
        return dict(kp=kp, vp=vp)
    old, new = _lengths(c)
    T, Hq, Hkv, D = s["T"], c["Hq"], c["Hkv"], c["D"]
    G, o = Hq // Hkv, torch.empty(T, Hq, D, dtype=torch.float64, device="cuda")
    lse, t0 = torch.empty(T, Hq, dtype=torch.float64, device="cuda"), 0
    for r, (a, n) in enumerate(zip(old, new)):
        ids = s["table"][r, : _blocks(a + n, page)].long()
        for g in range(Hkv):
            k = s["kp"][ids, g].reshape(-1, D)[: a + n].double()
            v = s["vp"][ids, g].reshape(-1, D)[: a + n].double()
            for h in range(g * G, g * G + G):
                for i0 in range(0, n, 1024):
                    i1 = min(n, i0 + 1024)
                    x = s["q"][t0 + i0:t0 + i1, h].double() @ k[: a + i1].T / math.sqrt(D)
                    late = torch.arange(a + i1, device="cuda") > torch.arange(a + i0, a + i1, device="cuda")[:, None]
                    x = x.masked_fill(late, -math.inf)
                    z = torch.logsumexp(x, 1)
                    lse[t0 + i0:t0 + i1, h] = z
                    o[t0 + i0:t0 + i1, h] = (x - z[:, None]).exp() @ v[: a + i1]
        t0 += n
    return dict(o=o, lse=lse)


def _exact_plan(c, s):
    """The definition, one token at a time, on the host."""
    old, new = _lengths(c)
    page, table, free, n = c["page"], s["table"].tolist(), s["free"].tolist(), int(s["n_free"])
    cu, kv_len, slots, pos, upto, left = [0], [], [], [], 0, n
    for r, (a, f) in enumerate(zip(old, new)):
        cu.append(cu[-1] + f)
        need = _blocks(a + f, page) - _blocks(a, page)
        upto += need
        if need and upto > n:
            kv_len.append(0)
            slots += [-1] * f
            pos += [-1] * f
            continue
        for i in range(need):
            left -= 1
            table[r][_blocks(a, page) + i] = free[left]
        kv_len.append(a + f)
        for p in range(a, a + f):
            slots.append(table[r][p // page] * page + p % page)
            pos.append(p)
    return dict(table=_ints(table), cu_q=_ints(cu), kv_len=_ints(kv_len), slots=_ints(slots), pos=_ints(pos), n_left=_ints([left]))
