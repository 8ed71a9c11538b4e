"""The paged calls on the GPU against their definitions (paged_ref.py): the plan and the write exactly, the attention
within the bound that its arithmetic allows."""
import importlib.util
import os
import random

import pytest
import torch

import paged_ref

lh = pytest.importorskip("paper_2605_06554_amd")

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32
BF, F32 = torch.bfloat16, torch.float32


def _i(x):
    return torch.tensor(x, dtype=I32, device=DEV)


# ------------------------------------------------------------------ plan

def _plan_case(R, page, width, T, pages, seed, short=1.0, odd=True, decode=False):
    rng = random.Random(seed)
    cached = [rng.choice([0, 1, page - 1, page, page + 1, rng.randrange(0, width * page)]) for _ in range(R)]
    fresh = [1 if decode else rng.choice([0, 1, 1, page, rng.randrange(0, 3 * page)]) for _ in range(R)]
    if odd:
        for _ in range(max(1, R // 8)):
            cached[rng.randrange(R)] = rng.choice([-1, width * page, width * page - 1])
            fresh[rng.randrange(R)] = rng.choice([-3, 0, width * page])
    ids = list(range(pages))
    rng.shuffle(ids)
    free = ids
    table = [[rng.randrange(-2, pages + 2) for _ in range(width)] for _ in range(R)]
    need = sum(paged_ref.blocks(max(c, 0) + max(f, 0), page) - paged_ref.blocks(max(c, 0), page) for c, f in zip(cached, fresh))
    n_free = min(pages, int(need * short))
    return cached, fresh, free, n_free, table, T if T else max(1, sum(max(f, 0) for f in fresh))


@pytest.mark.parametrize("R,page,width,T,pages,short", [
    (1, 16, 4, 0, 64, 1.0), (1, 16, 4, 5, 64, 1.0), (3, 16, 40, 200, 64, 1.0), (64, 16, 20, 0, 3000, 1.0),
    (64, 32, 20, 0, 3000, 0.5), (255, 16, 9, 0, 9000, 1.0), (256, 16, 9, 0, 9000, 0.9), (257, 128, 9, 70000, 9000, 1.0),
    (300, 1024, 3, 4000, 500, 0.7), (4096, 16, 5, 0, 30000, 0.99), (17, 64, 6, 100, 10, 3.0), (40, 16, 6, 0, 200, 0.0)])
def test_plan(R, page, width, T, pages, short):
    for seed in range(3):
        cached, fresh, free, n_free, table, Tn = _plan_case(R, page, width, T, pages, seed, short, seed > 0, seed == 2)
        print(f"[plan] R={R} page={page} width={width} T={Tn} pages={pages} n_free={n_free} seed={seed}", flush=True)
        pc = lh.paged(R, width, Tn, pages, page, 8, 2, 64)
        tab = _i(table)
        out = lh.page_plan(pc, _i(cached), _i(fresh), _i(free), _i([n_free]), tab)
        ref = paged_ref.plan(cached, fresh, free, n_free, table, page, pages, Tn)
        for name, got, want in zip(("table", "cu_q", "kv_len", "slots", "pos", "n_taken", "balance"),
                                   (tab, out["cu_q"], out["kv_len"], out["slots"], out["pos"], out["n_taken"], out["balance"]),
                                   (*ref[:5], [min(n_free, pages) - ref[5]], [ref[6]])):
            assert torch.equal(got.cpu(), torch.tensor(want, dtype=I32)), name


def test_plan_of_bad_pages_and_counts():
    """Page ids outside the pool (in the table and in the free list) give slots of -1 and go into the table as they
    are; a free count outside [0, pages] is taken as the nearest end."""
    print("[plan] bad pages", flush=True)
    pc = lh.paged(4, 4, 64, 8, 16, 2, 2, 64)
    table = [[8, -1, -1, -1], [-5, -1, -1, -1], [2, -1, -1, -1], [2 ** 31 - 1, -1, -1, -1]]
    for n_free in (100, -4, 8):
        args = [10, 3, 16, 20], [4, 30, 5, 1], [-1, 0, 1, 99, 2, -7, 3, 4], n_free
        tab = _i(table)
        out = lh.page_plan(pc, _i(args[0]), _i(args[1]), _i(args[2]), _i([n_free]), tab)
        ref = paged_ref.plan(*args, table, 16, 8, 64)
        for got, want in zip((tab, out["cu_q"], out["kv_len"], out["slots"], out["pos"]), ref):
            assert torch.equal(got.cpu(), torch.tensor(want, dtype=I32))
        assert int(out["n_taken"]) == min(max(n_free, 0), 8) - ref[5] and int(out["balance"]) == ref[6]


def test_plan_of_large_lengths():
    """Lengths whose sums pass 32 bits make their requests wait, and nothing else."""
    print("[plan] large lengths", flush=True)
    R, big = 6, 2 ** 31 - 1
    pc = lh.paged(R, 4, 40, 64, 16, 2, 2, 64)
    cached, fresh = [3, big, 0, 16, big, 1], [5, big, 4, 1, 1, 1]
    tab = _i([[9, -1, -1, -1]] * R)
    out = lh.page_plan(pc, _i(cached), _i(fresh), _i(list(range(64))), _i([64]), tab)
    ref = paged_ref.plan(cached, fresh, list(range(64)), 64, [[9, -1, -1, -1]] * R, 16, 64, 40)
    for got, want in zip((tab, out["cu_q"], out["kv_len"], out["slots"], out["pos"]), ref):
        assert torch.equal(got.cpu(), torch.tensor(want, dtype=I32))


def _timed_cases():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("timed_operators", at)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("spare", [1.3, 1.0, 0.9, 0.6, 0.2])
def test_plan_of_the_timed_ranges(spare):
    """The timed plans, and such with a pool that runs short, against their definition there; the pages left are
    n_free - n_taken (requests that need no page are admitted behind those that wait for some)."""
    m = _timed_cases()
    cases = [c for c in m.listed() if c["kind"] == "plan"]
    cases += [m._case("plan", R, (1, 300), (0, 5000), page=page, ones=0.5) for R, page in ((7, 16), (33, 64), (200, 256))]
    for c in cases:
        c = dict(c, spare=spare)
        print(f"[plan timed] R={c['R']} page={c['page']} spare={spare}", flush=True)
        s, want = m.prepare(c, 5), m.exact(c, 5)
        pc = lh.paged(c["R"], s["width"], s["T"], s["pages"], c["page"], c["Hq"], c["Hkv"], c["D"])
        out = lh.page_plan(pc, s["old"], s["new"], s["free"], s["n_free"], s["table"])
        got = dict(table=s["table"], n_left=s["n_free"] - out["n_taken"], **{n: out[n] for n in ("cu_q", "kv_len", "slots", "pos")})
        for name in want:
            assert torch.equal(got[name], want[name]), name


def test_every_free_page_is_handed_out():
    """A pool that runs short, over steps that go on with n_free - n_taken: a long request waits while others go on, and
    in the end no page is left."""
    print("[plan] every page", flush=True)
    page, pages, width, T = 16, 30, 40, 512
    pc = lh.paged(3, width, T, pages, page, 2, 2, 64)
    free, table = list(range(pages)), [[-1] * width for _ in range(3)]
    tab, n_free, cached = _i(table), pages, [0, 0, 0]
    ids, n_free_t = _i(free), _i([pages])
    for step in range(40):
        fresh = [15, 470 if step else 1, 1 if step < 16 else 0]
        out = lh.page_plan(pc, _i(cached), _i(fresh), ids, n_free_t, tab)
        table, _, kv, _, _, left, balance = paged_ref.plan(cached, fresh, free, n_free, table, page, pages, T)
        assert torch.equal(tab.cpu(), torch.tensor(table, dtype=I32)) and out["kv_len"].tolist() == kv
        n_free_t = n_free_t - out["n_taken"]
        n_free = left
        assert int(n_free_t) == left and (balance < left) == (step > 0)
        cached = [k or c for k, c in zip(kv, cached)]
    held = [i for r in range(3) for i in table[r][:paged_ref.blocks(cached[r], page)]]
    assert n_free == 0 and sorted(held) == free


# ------------------------------------------------------------------ write

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,Hkv,D,page,fused", [(1, 1, 64, 16, False), (7, 3, 64, 16, True), (130, 8, 128, 64, True),
                                                (1000, 2, 128, 1024, False), (33, 5, 64, 32, False)])
def test_write(T, Hkv, D, page, fused, dtype):
    print(f"[write] T={T} Hkv={Hkv} D={D} page={page} fused={fused} {dtype}", flush=True)
    g = torch.Generator(DEV).manual_seed(T)
    pages = T // page + 5
    pc = lh.paged(2, 8, T, pages, page, 2 * Hkv, Hkv, D, dtype)
    rows = torch.randn(T, 4 * Hkv, D, generator=g, device=DEV).to(dtype)
    k, v = rows[:, 2 * Hkv:3 * Hkv], rows[:, 3 * Hkv:]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:T].to(I32)
    slots[1::5] = -1
    if T > 3:
        slots[2], slots[3] = pages * page, 2 ** 31 - 1
    kp, vp = (torch.randn(pages, Hkv, page, D, generator=g, device=DEV).to(dtype) for _ in range(2))
    want = []
    for pool, x in ((kp, k), (vp, v)):
        w = pool.clone()
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                w[s // page, :, s % page] = x[t]
        want.append(w)
    lh.lh_page_write(pc, k, v, slots, kp, vp)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


# ------------------------------------------------------------------ attention

def _setup(lens, Hq, Hkv, D, page, dtype, seed=0, T=None, fused=False, trash=float("nan"), width=None, scale=1.0):
    """A step whose cache holds the requests' rows on scattered pages and `trash` everywhere else."""
    g = torch.Generator(DEV).manual_seed(1000 + seed)
    old, new = [a for a, _ in lens], [n for _, n in lens]
    total = [a + n for a, n in lens]
    held = [paged_ref.blocks(x, page) for x in total]
    pages = sum(held) + 3
    width = width or max(1, max(held)) + 1
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = [[-1] * width for _ in lens]
    kp, vp = (torch.full((pages, Hkv, page, D), trash, dtype=dtype, device=DEV) for _ in range(2))
    at = 0
    for r, n in enumerate(held):
        table[r][:n] = order[at:at + n]
        for b, page_id in enumerate(order[at:at + n]):
            m = min(page, total[r] - b * page)
            for pool in (kp, vp):
                pool[page_id, :, :m] = (scale * torch.randn(Hkv, m, D, generator=g, device=DEV)).to(dtype)
        at += n
    rows = sum(new)
    T = T or max(rows, 1)
    q = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device=DEV).to(dtype)[:, :Hq]
    q = q if fused else q.contiguous()
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    pc = lh.paged(len(lens), width, T, pages, page, Hq, Hkv, D, dtype)
    return dict(pc=pc, q=q, kp=kp, vp=vp, table=table, cu=cu, kv=total, page=page, rows=rows, T=T)


def _run(x, stream=None):
    pc = x["pc"]
    o = torch.full((x["T"], pc.Hq, pc.D), 7.0, dtype=x["q"].dtype, device=DEV)
    lse = torch.full((x["T"], pc.Hq), 7.0, device=DEV)
    ws = lh.paged_workspace(pc)
    ws.fill_(255)  # NaN patterns: nothing may be taken from an unwritten workspace
    lh.lh_sdpa_paged(pc, x["q"], x["kp"], x["vp"], _i(x["table"]), _i(x["cu"]), _i(x["kv"]), o, lse, ws, stream=stream)
    torch.cuda.synchronize()
    return o, lse


def _check(x, o, lse):
    ro, rl, to, tl = paged_ref.attend(x["q"], x["kp"], x["vp"], x["table"], x["cu"], x["kv"], x["page"])
    n = x["rows"]
    paged_ref.check("o", o[:n], ro[:n], to[:n])
    paged_ref.check("lse", lse[:n], rl[:n], tl[:n])
    assert bool((o[n:] == 7).all()) and bool((lse[n:] == 7).all()), "rows behind the last request were touched"


STEPS = {
    "one": [(0, 1)],
    "first_token_of_many": [(0, 1), (0, 1), (15, 1), (16, 1), (17, 1)],
    "decode": [(700, 1), (1, 1), (63, 1), (64, 1), (2500, 1), (127, 1), (31, 1)],
    "none_new": [(40, 0), (33, 1), (0, 0), (90, 0), (5, 2)],
    "drafts": [(100, 3), (1000, 5), (31, 2), (0, 4), (257, 6)],
    "chunk": [(300, 200)],
    "prompt": [(0, 333)],
    "prompts": [(0, 70), (0, 129), (0, 1), (0, 64)],
    "mixed": [(900, 1), (0, 150), (64, 64), (500, 1), (1, 1), (250, 31), (0, 0), (77, 1)],
    "long": [(9000, 1), (20000, 2)],
    "long_chunk": [(5000, 140), (12, 300)],
}


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", STEPS)
def test_attention(name, D, dtype):
    heads = {"one": (1, 1), "decode": (8, 2), "drafts": (6, 2), "mixed": (4, 1), "prompt": (3, 3), "long": (16, 2),
             "prompts": (10, 2)}.get(name, (4, 2))
    page = {"chunk": 64, "prompts": 32, "long": 128, "mixed": 16, "long_chunk": 256}.get(name, 16)
    print(f"[attend] {name} D={D} {dtype} heads={heads} page={page}", flush=True)
    x = _setup(STEPS[name], *heads, D, page, dtype, seed=len(name))
    _check(x, *_run(x))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (7, 1), (16, 1), (17, 1), (40, 2), (64, 1), (5, 5), (96, 6), (130, 1)])
@pytest.mark.parametrize("name", ["decode", "mixed"])
def test_attention_head_layouts(name, Hq, Hkv):
    print(f"[attend heads] {name} {Hq}/{Hkv}", flush=True)
    x = _setup(STEPS[name], Hq, Hkv, 64, 16, BF, seed=Hq)
    _check(x, *_run(x))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
def test_attention_page_sizes(page, dtype):
    print(f"[attend pages] {page} {dtype}", flush=True)
    for lens in ([(1500, 1), (page - 1, 1), (page, 1)], [(page - 1, 2 * page + 3), (0, page + 1), (1030, 90)]):
        x = _setup(lens, 4, 2, 128, page, dtype, seed=page)
        _check(x, *_run(x))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_fused_rows_and_padding(dtype):
    """q as a slice of a fused projection; more rows than the requests have (left as they were)."""
    print(f"[attend fused] {dtype}", flush=True)
    for name, more in (("decode", 9), ("mixed", 200), ("drafts", 1)):
        x = _setup(STEPS[name], 8, 2, 64, 16, dtype, seed=3, T=sum(n for _, n in STEPS[name]) + more, fused=True)
        _check(x, *_run(x))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", ["decode", "chunk"])
def test_rows_without_a_key(shape, dtype):
    """Requests that wait (kv_len 0) and chunks longer than the cache holds: their rows get 0 and -inf."""
    print(f"[attend empty] {shape} {dtype}", flush=True)
    lens = [(30, 1), (0, 1), (64, 1)] if shape == "decode" else [(40, 60), (0, 80), (10, 200), (5, 5)]
    x = _setup(lens, 4, 2, 64, 16, dtype, seed=8)
    x["kv"] = [31, 0, 65] if shape == "decode" else [100, 0, 130, 3]
    o, lse = _run(x)
    _check(x, o, lse)
    a = x["cu"][1]
    assert bool((o[a:x["cu"][2]] == 0).all()) and bool((lse[a:x["cu"][2]] == -float("inf")).all())


@pytest.mark.parametrize("R,new,Hq,Hkv,dtype", [(700, (0, 1), 4, 2, BF), (4096, (1, 1), 2, 2, F32), (600, (4, 20), 16, 1, BF),
                                                (900, (20, 40), 8, 1, BF), (300, (1, 5), 8, 2, F32)])
def test_more_requests_than_threads(R, new, Hq, Hkv, dtype):
    """The cut of the work sums over the requests a workgroup's threads at a time."""
    print(f"[attend many] R={R} new={new} {Hq}/{Hkv} {dtype}", flush=True)
    rng = random.Random(R)
    lens = [(rng.choice([0, 3, 16, rng.randrange(60)]), rng.randint(*new)) for _ in range(R)]
    x = _setup(lens, Hq, Hkv, 64, 16, dtype, seed=R)
    _check(x, *_run(x))


@pytest.mark.parametrize("D,dtype", [(128, BF), (64, BF), (128, F32)])
def test_random_steps(D, dtype):
    """Lengths, heads and pages at random: every variant of the kernels and tiles that parts divide anywhere."""
    rng = random.Random(D + (dtype == F32))
    for i in range(14):
        Hkv = rng.choice([1, 2, 3])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 6, 8])
        most = rng.choice([1, 2, 8, 40, 200, 500])
        lens = [(rng.choice([0, 1, 15, 64, rng.randrange(3000)]), rng.choice([0, 1, 1, most, rng.randint(1, most)]))
                for _ in range(rng.choice([1, 2, 5, 12, 30]))]
        page = rng.choice([16, 32, 64, 128])
        print(f"[attend random] {i} D={D} {dtype} {Hq}/{Hkv} page={page} lens={lens}", flush=True)
        x = _setup(lens, Hq, Hkv, D, page, dtype, seed=i, fused=rng.random() < 0.5)
        _check(x, *_run(x))


def test_without_lse():
    print("[attend] no lse", flush=True)
    for name in ("decode", "mixed"):
        x = _setup(STEPS[name], 8, 2, 64, 16, BF, seed=61)
        o, _ = _run(x)
        o2 = torch.full_like(o, 7.0)
        lh.lh_sdpa_paged(x["pc"], x["q"], x["kp"], x["vp"], _i(x["table"]), _i(x["cu"]), _i(x["kv"]), o2, None,
                         lh.paged_workspace(x["pc"]))
        assert torch.equal(o, o2)


def test_step_without_rows():
    print("[attend] no rows", flush=True)
    x = _setup([(20, 0), (0, 0)], 4, 2, 64, 16, BF, T=5)
    _check(x, *_run(x))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("lens", [[(100, 150)], [(37, 5), (500, 1)], [(0, 400), (3000, 20)]])
def test_a_rows_odd_values_reach_no_earlier_row(lens, bad, dtype):
    """K and V of a chunk's later token hold NaN or infinities: the rows before it do not see them, and other requests
    do not either."""
    print(f"[attend odd] {lens} {bad} {dtype}", flush=True)
    x = _setup(lens, 4, 2, 64, 16, dtype, seed=11)
    clean_o, clean_l = _run(x)
    a, n = lens[0]
    p = a + n - (n // 3) - 1  # position of the odd token
    page_id, off = x["table"][0][p // 16], p % 16
    for pool in ("kp", "vp"):
        y = dict(x, **{pool: x[pool].clone()})
        y[pool][page_id, 0, off, 5] = bad
        o, lse = _run(y)
        rows = torch.arange(x["T"], device=DEV)
        before = (rows < p - a) | (rows >= n)
        assert torch.equal(o[before], clean_o[before]) and torch.equal(lse[before], clean_l[before])
        after = ~before
        assert torch.equal(o[after][:, 2:], clean_o[after][:, 2:])  # the other KV head
        if pool == "vp":
            assert torch.equal(lse, clean_l)
            hit = o[after][:, :2, 5]
            assert not bool(torch.isfinite(hit).any())
            rest = [d for d in range(64) if d != 5]
            assert torch.equal(o[:, :, rest], clean_o[:, :, rest])
        elif bad != bad:
            assert bool(torch.isnan(o[after][:, :2]).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[(300, 1)], [(300, 1), (40, 0), (5000, 3)], [(300, 9), (20, 7)], [(300, 40), (100, 1)],
                                  [(300, 200), (700, 1), (64, 100)]])
def test_infinite_values_that_rows_see(lens, dtype):
    """Infinities and NaN of V among the first keys, which all rows see: their columns hold what the sum over the keys
    does (one sign: that infinity; both, or NaN: NaN), the others are as they were."""
    print(f"[attend seen odd] {lens} {dtype}", flush=True)
    for D, Hq in ((64, 4), (128, 8)):
        x = _setup(lens, Hq, 2, D, 16, dtype, seed=31)
        x["q"] = x["q"] * 0.25  # logits of a few units: no weight vanishes
        clean, _ = _run(x)
        inf = float("inf")
        for r in range(len(lens)):
            page = x["vp"][x["table"][r][0]]
            for key, col, bad in ((3, 0, inf), (5, 1, -inf), (9, 2, float("nan")), (2, 3, inf), (15, 3, -inf), (4, D - 1, inf), (12, D - 1, inf)):
                page[1, key, col] = bad
        o, lse = _run(x)
        _check(x, o, lse)
        half = Hq // 2
        assert torch.equal(o[:, :half], clean[:, :half]) and torch.equal(o[:, :, 4:D - 1], clean[:, :, 4:D - 1])
        assert bool((o[:x["rows"], half:, 0] == inf).all()) and bool((o[:x["rows"], half:, 1] == -inf).all())
        assert bool(torch.isnan(o[:x["rows"], half:, 2:4]).all()) and bool((o[:x["rows"], half:, D - 1] == inf).all())


def _waves(T, G, R):
    """Waves of a workgroup of the tile kernel (bf16) for a step's rows a request."""
    rows = T * G // R
    assert rows > 32
    wide = rows > 256 and -(-rows // 384) * 384 * 32 <= -(-rows // 256) * 256 * 33
    return 4 if rows <= 112 else 12 if wide else 8


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("waves,chunk", [(4, 261), (8, 901), (12, 1349)])
def test_odd_values_in_the_last_keys_of_small_tiles(waves, chunk, D, bad):
    """A chunk whose last tile has 10 rows, beside requests of one to three tokens whose last block of 32 keys falls to
    each wave in turn: a value of V among the last keys that is not finite reaches the rows that see its key, in
    its column, and nothing else."""
    print(f"[attend odd, small tiles] {waves} waves D={D} {bad}", flush=True)
    for first in (0, 8):  # blocks before the last one
        small = [(32 * (first + i) + (3, 29, 15, 20)[i % 4], 1 + i % 3) for i in range(8)]
        lens = [(300, chunk)] + small
        assert _waves(sum(n for _, n in lens), 2, len(lens)) == waves and chunk * 2 % (32 * waves) == 10
        x = _setup(lens, 4, 2, D, 16, BF, seed=61 + first)
        clean_o, clean_l = _run(x)
        y, col = dict(x, vp=x["vp"].clone()), 5
        sees = torch.zeros(x["T"], dtype=torch.bool, device=DEV)
        for r, (old, n) in enumerate(lens):
            p = old + n - 1 - (3 if r == 0 else 1 if n == 3 else 0)
            y["vp"][x["table"][r][p // 16], 0, p % 16, col] = bad
            sees[x["cu"][r] + p - old:x["cu"][r + 1]] = True
        want = clean_o.clone()
        want[sees, :2, col] = bad
        for again in range(3):
            o, lse = _run(y)
            same = (o == want) | (torch.isnan(o) & torch.isnan(want))
            assert bool(same.all()), f"{int((~same).sum())} elements, first {tuple(map(int, (~same).nonzero()[0]))}"
            assert torch.equal(lse, clean_l)


def test_large_logits():
    """Logits in the thousands, where a weight is 0 or 1, and runs of growing maxima."""
    print("[attend large logits]", flush=True)
    for dtype in (BF, F32):
        x = _setup([(900, 1), (200, 120)], 4, 2, 128, 16, dtype, seed=21, scale=60.0)
        x["q"] = (x["q"].float() * 8).to(dtype)
        _check(x, *_run(x))
        x = _setup([(1500, 1), (600, 60)], 2, 2, 64, 32, dtype, seed=22)
        x["q"] = x["q"].float().abs().to(dtype)
        for r in range(2):  # keys grow along the request
            for b, page_id in enumerate(x["table"][r]):
                if page_id >= 0:
                    x["kp"][page_id] = (x["kp"][page_id].float().abs() * (0.01 * (b + 1))).to(dtype)
        _check(x, *_run(x))


def test_bad_tables_and_lengths_stay_in_bounds():
    """Page ids outside the pool, lengths beyond the table and offsets in disorder are clamped: the other requests'
    results are theirs all the same."""
    print("[attend bad tables]", flush=True)
    for lens in ([(300, 1), (200, 1), (90, 1)], [(300, 20), (200, 100), (90, 70)]):
        x = _setup(lens, 4, 2, 64, 16, BF, seed=31, trash=1.0)
        o, lse = _run(x)
        y = dict(x, table=[list(t) for t in x["table"]], kv=list(x["kv"]))
        y["table"][1] = [2 ** 31 - 1, -2 ** 31, 5000] * 20
        y["table"][1] = y["table"][1][:len(x["table"][1])]
        y["kv"][1] = 2 ** 31 - 1
        o2, lse2 = _run(y)
        keep = torch.ones(x["T"], dtype=torch.bool, device=DEV)
        keep[x["cu"][1]:x["cu"][2]] = False
        # the split of the work follows the lengths, so the sums' order may differ: within both runs' bounds
        _, _, to, tl = paged_ref.attend(x["q"], x["kp"], x["vp"], x["table"], x["cu"], x["kv"], 16)
        paged_ref.check("o", o2[keep], o[keep].double(), 2 * to[keep])
        paged_ref.check("lse", lse2[keep], lse[keep].double(), 2 * tl[keep])
        z = dict(x, cu=[-5, 10 ** 9, -3, 4])
        _run(z)


def test_same_call_same_bits_on_another_stream():
    print("[attend bits]", flush=True)
    for name in ("decode", "mixed", "long_chunk"):
        x = _setup(STEPS[name], 8, 2, 128, 16, BF, seed=41)
        o, lse = _run(x)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for stream in (None, s):
            o2, lse2 = _run(x, stream)
            assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_helpers_on_another_stream():
    """page_plan and attention_paged with a stream of their own (as an object, its address, and the null stream's) and
    a workspace that they allocate: the results are the default stream's, also where memory freed there is taken again at once."""
    print("[attend] helpers on another stream", flush=True)
    R, page, Hq, Hkv, D = 5, 16, 8, 2, 64
    cached, fresh = [0] * R, [40, 1, 300, 17, 64]
    T, pages, width = sum(fresh), 40, 20
    pc = lh.paged(R, width, T, pages, page, Hq, Hkv, D)
    g = torch.Generator(DEV).manual_seed(5)
    q, k, v = (torch.randn(T, h, D, generator=g, device=DEV).to(BF) for h in (Hq, Hkv, Hkv))
    args = _i(cached), _i(fresh), _i(list(range(pages))), _i([pages])
    side = torch.cuda.Stream()
    outs = []
    for stream in (None, side, side.cuda_stream, 0):
        table = torch.full((R, width), -1, dtype=I32, device=DEV)
        kp, vp = lh.paged_cache(pages, page, Hkv, D)
        torch.cuda.synchronize()
        plan = lh.page_plan(pc, *args, table, stream=stream)
        for _ in range(3):
            o, lse = lh.attention_paged(pc, q, k, v, kp, vp, table, plan, stream=stream)
            torch.full((1 << 24,), 255, dtype=torch.uint8, device=DEV)  # (takes what the default stream has free)
        torch.cuda.synchronize()
        outs.append((o.clone(), lse.clone(), table.clone()))
    assert bool(torch.isfinite(outs[0][0].float()).all())
    for got in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got, outs[0]))


def test_pool_beyond_32_bit_offsets():
    """A pool of more than 2^32 bytes (and elements past 2^31): a request on its last pages."""
    print("[attend large pool]", flush=True)
    Hkv, page, D = 8, 64, 128
    pages = 2 ** 31 // (Hkv * page * D) + 9
    kp, vp = (torch.empty(pages, Hkv, page, D, dtype=BF, device=DEV) for _ in range(2))
    used = [pages - 1, 0, pages - 5, pages - 2]
    lens = [(page + 9, 1), (100, 1)]
    g = torch.Generator(DEV).manual_seed(2)
    for p in used:
        kp[p], vp[p] = (torch.randn(Hkv, page, D, generator=g, device=DEV).to(BF) for _ in range(2))
    for new in (1, 70):
        table = [used[:2], used[2:]]
        total = [a + 1 for a, _ in lens]
        T = 2 * new
        pc = lh.paged(2, 2, T, pages, page, 16, Hkv, D)
        q = torch.randn(T, 16, D, generator=g, device=DEV).to(BF)
        k, v = (torch.randn(T, Hkv, D, generator=g, device=DEV).to(BF) for _ in range(2))
        slots = [[table[r][p // page] * page + p % page for p in range(total[r] - new, total[r])] for r in range(2)]
        lh.lh_page_write(pc, k, v, _i(slots[0] + slots[1]), kp, vp)
        x = dict(pc=pc, q=q, kp=kp, vp=vp, table=table, cu=[0, new, T], kv=total, page=page, rows=T, T=T)
        for r in range(2):
            p = total[r] - 1
            assert torch.equal(kp[table[r][p // page], :, p % page], k[r * new + new - 1])
        _check(x, *_run(x))


# ------------------------------------------------------------------ together

def _serve(pc, state, q, k, v, cached, fresh, ws):
    plan = lh.page_plan(pc, _i(cached), _i(fresh), state["free"], state["n_free"], state["table"])
    o, lse = lh.attention_paged(pc, q, k, v, state["kp"], state["vp"], state["table"], plan, ws)
    state["n_free"] = state["n_free"] - plan["n_taken"]
    return plan, o, lse


@pytest.mark.parametrize("dtype,T,Hq,Hkv,new", [(BF, 300000, 64, 2, 75), (F32, 280000, 64, 64, 70)])
def test_rows_beyond_32_bit_offsets(dtype, T, Hq, Hkv, new):
    """More than 2^31 elements of q and o: the first and the last requests' rows against the definition."""
    print(f"[attend] rows beyond 32-bit offsets {dtype}", flush=True)
    D, page, R = 128, 128, T // new
    assert T * Hq * D > 2 ** 31 and R * new == T
    g = torch.Generator(DEV).manual_seed(3)
    pc = lh.paged(R, 1, T, R, page, Hq, Hkv, D, dtype)
    q = torch.empty(T, Hq, D, dtype=dtype, device=DEV).normal_(generator=g)
    kp, vp = (torch.empty(R, Hkv, page, D, dtype=dtype, device=DEV).normal_(generator=g) for _ in range(2))
    table = torch.arange(R - 1, -1, -1, dtype=I32, device=DEV)[:, None].contiguous()
    cu, kv = torch.arange(0, T + 1, new, dtype=I32, device=DEV), torch.full((R,), new + 10, dtype=I32, device=DEV)
    o, lse = torch.full((T, Hq, D), 7.0, dtype=dtype, device=DEV), torch.full((T, Hq), 7.0, device=DEV)
    lh.lh_sdpa_paged(pc, q, kp, vp, table, cu, kv, o, lse, lh.paged_workspace(pc))
    torch.cuda.synchronize()
    for r in (0, R // 2, R - 1):
        a, b = r * new, r * new + new
        ref = paged_ref.attend(q[a:b], kp, vp, [[R - 1 - r]], [0, new], [new + 10], page)
        paged_ref.check("o", o[a:b], ref[0], ref[2])
        paged_ref.check("lse", lse[a:b], ref[1], ref[3])
    assert bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_requests_that_share_pages(dtype):
    """Requests whose tables name the same pages (a common beginning), and one page twice in a table: each reads them as
    its own."""
    print(f"[attend] shared pages {dtype}", flush=True)
    for lens in ([(100, 1), (90, 1), (200, 3)], [(100, 60), (90, 1), (200, 150)]):
        x = _setup(lens, 4, 2, 64, 16, dtype, seed=51)
        for r in (1, 2):
            x["table"][r][:4] = x["table"][0][:4]
        x["table"][2][6] = x["table"][2][5]
        _check(x, *_run(x))


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [(BF, 8, 2, 128, 16), (F32, 4, 4, 64, 32)])
def test_serving_steps_match_whole_sequences(dtype, Hq, Hkv, D, page):
    """Three requests served in steps of chunks, drafts and single tokens (one joins late, one waits for pages once)
    against causal attention over each whole sequence; prompts also against lh_sdpa_fwd."""
    print(f"[serve] {dtype} {Hq}/{Hkv} D={D} page={page}", flush=True)
    g = torch.Generator(DEV).manual_seed(77)
    lens = [230, 75, 140]
    full = [[torch.randn(n, H, D, generator=g, device=DEV).to(dtype) for H in (Hq, Hkv, Hkv)] for n in lens]
    steps = [[100, 30, 0], [1, 1, 0], [64, 1, 90], [60, 40, 1], [4, 2, 48], [1, 1, 1]]
    pages = sum(paged_ref.blocks(n, page) for n in lens) + 1
    width = paged_ref.blocks(max(lens), page)
    table = torch.full((3, width), -1, dtype=I32, device=DEV)
    kp, vp = lh.paged_cache(pages, page, Hkv, D, dtype)
    kp.fill_(float("nan")), vp.fill_(float("nan"))
    state = dict(free=torch.randperm(pages, generator=g, device=DEV).to(I32), n_free=_i([pages]), table=table, kp=kp, vp=vp)
    cached, outs = [0, 0, 0], [[], [], []]
    for fresh in steps:
        T = sum(fresh) + 3
        pc = lh.paged(3, width, T, pages, page, Hq, Hkv, D, dtype)
        rows = [torch.cat([full[r][i][cached[r]:cached[r] + fresh[r]] for r in range(3)] + [torch.zeros(3, H, D, dtype=dtype, device=DEV)])
                for i, H in enumerate((Hq, Hkv, Hkv))]
        plan, o, lse = _serve(pc, state, *rows, cached, fresh, lh.paged_workspace(pc))
        cu = plan["cu_q"].tolist()
        assert plan["kv_len"].tolist() == [c + f for c, f in zip(cached, fresh)]
        for r in range(3):
            outs[r].append((o[cu[r]:cu[r + 1]], lse[cu[r]:cu[r + 1]]))
            cached[r] += fresh[r]
    assert cached == lens
    for r in range(3):
        n = cached[r]
        m = paged_ref.blocks(n, page)
        k, v = (torch.zeros(m, Hkv, page, D, dtype=dtype, device=DEV) for _ in range(2))
        for pool, x in ((k, full[r][1]), (v, full[r][2])):
            for p in range(n):
                pool[p // page, :, p % page] = x[p]
        ro, rl, to, tl = paged_ref.attend(full[r][0][:n], k, v, [list(range(m))], [0, n], [n], page)
        paged_ref.check("o", torch.cat([a for a, _ in outs[r]]), ro, to)
        paged_ref.check("lse", torch.cat([b for _, b in outs[r]]), rl, tl)
        if Hq == Hkv:  # the layer's own causal attention, L = 1, on the same rows
            pr = lh.problem(1, n, Hq, Hkv, D, 2, 1, 0, dtype)
            x = [t[:n].transpose(0, 1).contiguous()[None] for t in full[r]]
            os_, l2 = torch.empty_like(x[0]), torch.empty(1, Hq, n, device=DEV)
            lh.lh_sdpa_fwd(pr, *x, os_, l2)
            paged_ref.check("lh_sdpa_fwd", os_[0].transpose(0, 1), ro, to)


def test_captured_steps_replay_with_other_lengths():
    """Plan, write and attention of a step captured once; replayed with other lengths, rows and tables in the same
    buffers, with eager work between, against eager calls bit for bit."""
    print("[graph]", flush=True)
    R, width, T, pages, page, Hq, Hkv, D = 5, 40, 96, 220, 16, 8, 2, 64
    pc = lh.paged(R, width, T, pages, page, Hq, Hkv, D)
    g = torch.Generator(DEV).manual_seed(5)
    e = lambda *s, dt=I32: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
    b = dict(cached=e(R), fresh=e(R), free=e(pages), n_free=e(1), table=e(R, width), cu=e(R + 1), kv=e(R), slots=e(T), pos=e(T),
             left=e(1), q=e(T, Hq, D, dt=BF), k=e(T, Hkv, D, dt=BF), v=e(T, Hkv, D, dt=BF), kp=e(pages, Hkv, page, D, dt=BF),
             vp=e(pages, Hkv, page, D, dt=BF), o=e(T, Hq, D, dt=BF), lse=e(T, Hq, dt=F32))
    ws = lh.paged_workspace(pc)

    def step(b, ws):
        lh.lh_page_plan(pc, b["cached"], b["fresh"], b["free"], b["n_free"], b["table"], b["cu"], b["kv"], b["slots"], b["pos"], b["left"])
        lh.lh_page_write(pc, b["k"], b["v"], b["slots"], b["kp"], b["vp"])
        lh.lh_sdpa_paged(pc, b["q"], b["kp"], b["vp"], b["table"], b["cu"], b["kv"], b["o"], b["lse"], ws)

    def fill(seed):
        rng = random.Random(seed)
        cached = [rng.choice([0, 15, 16, rng.randrange(500)]) for _ in range(R)]
        fresh = [rng.choice([0, 1, rng.randrange(1, 40)]) for _ in range(R)] if seed % 2 else [1] * R
        while sum(fresh) > T:
            fresh[fresh.index(max(fresh))] = 1
        ids = list(range(pages))
        rng.shuffle(ids)
        table, at = [[-1] * width for _ in range(R)], 0
        for r in range(R):
            m = paged_ref.blocks(cached[r], page)
            table[r][:m] = ids[at:at + m]
            at += m
        free = ids[at:]
        x = dict(cached=_i(cached), fresh=_i(fresh), free=_i(free + [-1] * (pages - len(free))), n_free=_i([len(free)]), table=_i(table))
        for n in ("q", "k", "v", "kp", "vp"):
            x[n] = torch.randn(b[n].shape, generator=g, device=DEV).to(BF)
        return x, sum(fresh)

    sets = [fill(s) for s in (1, 2, 3)]
    keys = ("table", "cu", "kv", "slots", "pos", "left", "kp", "vp", "o", "lse")
    refs = []
    for x, _ in sets:
        y = {n: x[n].clone() if n in x else torch.zeros_like(b[n]) for n in b}
        step(y, lh.paged_workspace(pc))
        torch.cuda.synchronize()
        refs.append(y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(b, ws)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b, ws)
    for rep, which in enumerate((0, 1, 0, 2, 1, 2)):
        for n, t in sets[which][0].items():
            b[n].copy_(t)
        b["o"].zero_(), b["lse"].zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in keys:
            assert torch.equal(b[n], refs[which][n]), f"replay {rep} (step {which}): {n}"


def test_two_steps_at_once():
    """Two steps in flight on two streams, each with its own workspace."""
    print("[two streams]", flush=True)
    xs = [_setup(STEPS["decode"], 8, 2, 128, 16, BF, seed=51), _setup(STEPS["long_chunk"], 8, 2, 128, 16, BF, seed=52)]
    refs = [_run(x) for x in xs]
    outs, streams = [], [torch.cuda.Stream() for _ in xs]
    bufs = []
    for x in xs:
        pc = x["pc"]
        bufs.append((torch.empty(x["T"], pc.Hq, pc.D, dtype=BF, device=DEV), torch.empty(x["T"], pc.Hq, device=DEV), lh.paged_workspace(pc),
                     _i(x["table"]), _i(x["cu"]), _i(x["kv"])))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, (o, lse, ws, t, c, n) in zip(xs, streams, bufs):
            lh.lh_sdpa_paged(x["pc"], x["q"], x["kp"], x["vp"], t, c, n, o, lse, ws, stream=s)
    torch.cuda.synchronize()
    for (o, lse, *_), (ro, rl), x in zip(bufs, refs, xs):
        assert torch.equal(o[:x["rows"]], ro[:x["rows"]]) and torch.equal(lse[:x["rows"]], rl[:x["rows"]])


def test_two_graphs_share_a_workspace():
    """Two captured steps with one workspace, replayed in turn: nothing of one call is left for another."""
    print("[two graphs]", flush=True)
    xs = [_setup(STEPS["decode"], 8, 2, 128, 16, BF, seed=71), _setup(STEPS["mixed"], 8, 2, 128, 16, BF, seed=72)]
    refs = [_run(x) for x in xs]
    need = max(lh.lh_paged_workspace_bytes(x["pc"]) for x in xs)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for x in xs:
        pc = x["pc"]
        args = (_i(x["table"]), _i(x["cu"]), _i(x["kv"]), torch.empty(x["T"], pc.Hq, pc.D, dtype=BF, device=DEV),
                torch.empty(x["T"], pc.Hq, device=DEV), ws)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            lh.lh_sdpa_paged(pc, x["q"], x["kp"], x["vp"], *args)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lh.lh_sdpa_paged(pc, x["q"], x["kp"], x["vp"], *args)
        graphs.append(g), outs.append(args)
    for rep in range(4):
        for g, args, (ro, rl), x in zip(graphs, outs, refs, xs):
            args[3].zero_(), args[4].zero_()
            g.replay()
            torch.cuda.synchronize()
            n = x["rows"]
            assert torch.equal(args[3][:n], ro[:n]) and torch.equal(args[4][:n], rl[:n]), f"replay {rep}"
