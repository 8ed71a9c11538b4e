"""The paged calls' refusals, on the host: nothing is launched by any of them."""
import ctypes
import random

import pytest
import torch

import paged_ref
import paper_2605_06554_amd as lh


def _pc(**kw):
    base = dict(R=4, max_blocks=8, T=100, pages=64, page=16, Hq=8, Hkv=2, D=64, dtype=lh.LH_BF16)
    base.update(kw)
    return lh.paged(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0),
    (dict(R=0), -2), (dict(R=4096), 0), (dict(R=4097), -2),
    (dict(T=0), -2), (dict(pages=0), -2), (dict(max_blocks=0), -2),
    (dict(page=8), -3), (dict(page=24), -3), (dict(page=1024), 0), (dict(page=2048), -3), (dict(page=-16), -3),
    (dict(Hq=3), -3), (dict(Hkv=0), -3), (dict(Hq=0, Hkv=1), -3), (dict(D=96), -3), (dict(D=0), -3),
    (dict(dtype=2), -4), (dict(dtype=torch.float32), 0),
    (dict(scale=float("nan")), -8), (dict(scale=float("inf")), -8), (dict(scale=-1.0), -3), (dict(scale=0.5), 0),
    (dict(pages=2 ** 27 - 1), 0), (dict(pages=2 ** 27), -2),          # pages * page < 2^31
    (dict(max_blocks=2 ** 26), 0), (dict(max_blocks=2 ** 26 + 1), -2),  # max_blocks * page <= 2^30
    (dict(T=2 ** 27), 0), (dict(T=2 ** 27 + 1), -2),                  # T * Hq <= 2^30
    (dict(R=16, T=2 ** 27 - 4, max_blocks=2 ** 24), -2),              # 2^34 (2^28 + 2^27) > 2^62 units of the cut
    (dict(R=8, T=2 ** 27 - 4, max_blocks=2 ** 24), 0),
    (dict(R=4096, T=2 ** 27, max_blocks=2 ** 26), -2), (dict(R=4096, T=8192, Hq=32, Hkv=8, max_blocks=2 ** 26), 0),
])
def test_check_codes(kw, code):
    pc = _pc(**kw)
    assert lh.lh_paged_check(pc) == code
    if code:
        assert lh.lh_last_error() != ""
        with pytest.raises(lh.LighthouseError):
            lh.lh_paged_workspace_bytes(pc)
    else:
        assert lh.lh_paged_workspace_bytes(pc) >= 0


def _units(pc, TM):
    """The units of the cut (csrc/lh_paged_sdpa.h: Req) where every request's rows are clipped to all T and its keys to all
    that its table row holds, in exact integers; lastw and the constant at their largest."""
    G = pc.Hq // pc.Hkv
    past, step, over = pc.max_blocks * pc.page, TM // G if G < TM else 1, 160
    tiles = -(-pc.T * G // TM)
    before = 16 * ((tiles - 1) * (past + over) + step * (tiles - 1) * tiles // 2)
    return pc.R * pc.Hkv * (before + 16 * (past + tiles * step + over))


@pytest.mark.parametrize("kw,code", [
    (dict(R=4096, T=2 ** 14, Hq=2 ** 16, Hkv=1, max_blocks=1, dtype=torch.float32), -2),  # 2^25 tiles a request: 2^65 units
    (dict(R=4096, T=2 ** 14, Hq=2 ** 16, Hkv=1, max_blocks=1), -2),
    (dict(R=4096, T=2 ** 20, Hq=2 ** 10, Hkv=2, max_blocks=1), -2),
    (dict(R=1, T=2 ** 14, Hq=2 ** 16, Hkv=1, max_blocks=1, dtype=torch.float32), 0),
    (dict(R=4096, T=4096, Hq=128, Hkv=1, max_blocks=2 ** 18), 0),
    (dict(R=4096, T=2 ** 16, Hq=64, Hkv=1, max_blocks=2 ** 16), 0),
])
def test_units_of_the_cut_fit_64_bits(kw, code):
    pc = _pc(**kw)
    assert lh.lh_paged_check(pc) == code
    if code == 0:
        assert max(_units(pc, TM) for TM in (16, 32, 128, 256, 384)) < 2 ** 63


def test_units_of_the_cut_fit_64_bits_wherever_the_check_passes():
    rng = random.Random(9)
    passed = near = 0
    for _ in range(20000):
        two = lambda hi: 2 ** rng.uniform(0, hi)  # noqa: E731
        Hkv = int(two(8))
        pc = _pc(R=int(two(12)), T=int(two(30)), Hkv=Hkv, Hq=Hkv * int(two(18)), max_blocks=int(two(26)))
        if lh.lh_paged_check(pc) == 0:
            most = max(_units(pc, TM) for TM in (16, 32, 128, 256, 384))
            assert most < 2 ** 63, (pc, most)
            passed, near = passed + 1, near + (most > 2 ** 58)
    assert passed > 3000 and near > 20, (passed, near)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 8, 128), (8, 2, 64), (32, 8, 128), (64, 1, 128), (400, 1, 64)])
def test_a_workspace_serves_smaller_steps(Hq, Hkv, D, dtype):
    """One workspace for the largest R and T: no step of fewer requests or rows needs more."""
    sizes = lambda: [1, 2, 3, 4, 7, 8, 9, 16, 32, 33, 64, 96, 97, 128, 256, 257, 384, 512, 1000, 4096]  # noqa: E731
    need = {(R, T): lh.lh_paged_workspace_bytes(_pc(R=R, T=T, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype)) for R in sizes() for T in sizes()}
    for a, b in zip(sizes(), sizes()[1:]):
        for x in sizes():
            assert need[a, x] <= need[b, x] and need[x, a] <= need[x, b], (a, b, x)
    assert max(need.values()) <= 103 << 20


def test_null_and_misaligned_pointers():
    lib, pc = lh._load(), _pc()
    ok = [0x10000 * (i + 1) for i in range(12)]
    by = ctypes.byref(pc)
    assert lib.lh_paged_check(None) == -1
    assert lib.lh_paged_workspace_bytes(by, None) == -1
    for i in range(10):  # each pointer of the plan in turn
        bad = ok[:10]
        bad[i] = None
        assert lib.lh_page_plan(by, *bad, ok[10], None) == -1
        bad[i] = 0x10002
        assert lib.lh_page_plan(by, *bad, None, None) == -5
    assert lib.lh_page_plan(by, *ok[:10], 0x10001, None) == -5
    row = 2 * 64
    for args, code in [((None, row, 0x1000, row, 0x2000, 0x3000, 0x4000), -1),
                       ((0x1008, row, 0x1000, row, 0x2000, 0x3000, 0x4000), -5),
                       ((0x1000, row, 0x1000, row, 0x2002, 0x3000, 0x4000), -5),
                       ((0x1000, row, 0x1000, row, 0x2000, 0x3000, 0x4008), -5),
                       ((0x1000, row - 8, 0x1000, row, 0x2000, 0x3000, 0x4000), -2),
                       ((0x1000, row, 0x1000, row + 4, 0x2000, 0x3000, 0x4000), -5),
                       ((0x1000, row, 0x1000, 2 ** 41, 0x2000, 0x3000, 0x4000), -2),
                       ((0x1000, 0, 0x1000, row, 0x2000, 0x3000, 0x4000), -2),
                       ((0x1000, -row, 0x1000, row, 0x2000, 0x3000, 0x4000), -2)]:
        assert lib.lh_page_write(by, *args, None) == code, (args, lh.lh_last_error())
    need = lh.lh_paged_workspace_bytes(pc)
    good = [0x1000, 8 * 64, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x10000, need]
    for i, value, code in [(0, None, -1), (0, 0x1008, -5), (1, 8 * 64 - 8, -2), (1, 8 * 64 + 1, -5), (2, None, -1),
                           (3, 0x3004, -5), (4, None, -1), (4, 0x4002, -5), (5, None, -1), (6, 0x6001, -5),
                           (7, None, -1), (7, 0x7008, -5), (8, 0x8002, -5)]:
        bad = list(good)
        bad[i] = value
        assert lib.lh_sdpa_paged(by, *bad, None) == code, (i, value, lh.lh_last_error())
    if need:
        for i, value, code in [(9, None, -6), (9, 0x10010, -5), (10, need - 1, -6)]:
            bad = list(good)
            bad[i] = value
            assert lib.lh_sdpa_paged(by, *bad, None) == code
    assert lib.lh_sdpa_paged(ctypes.byref(_pc(D=32)), *good, None) == -3


def test_overlapping_arrays():
    """An output that shares memory with another array of its call is refused; inputs may share theirs."""
    lib, pc = lh._load(), _pc()
    by = ctypes.byref(pc)
    size = [16, 16, 256, 4, 128, 20, 16, 400, 400, 4, 4]  # bytes of the plan's arrays; the last seven are outputs
    at, good = 1 << 20, []
    for n in size:
        good.append(at)
        at += n
    for i in range(4, 11):
        for j in range(i):
            for where in (good[j] + size[j] - 4, good[j] - size[i] + 4):  # the last word of it, and the first
                bad = list(good)
                bad[i] = where
                assert lib.lh_page_plan(by, *bad, None) == -3 and "overlap" in lh.lh_last_error(), (i, j)
    row, rows, pool = 2 * 64, 100 * 2 * 64 * 2, 64 * 2 * 16 * 64 * 2
    M = 1 << 24
    k, v, slots, kp, vp = M, 2 * M, 3 * M, 4 * M, 5 * M
    for a in ((k, v, slots, kp, kp), (k, v, slots, kp, kp + pool - 16), (k, v, slots, k + rows - 16, vp), (k, v, slots, k - pool + 16, vp),
              (k, v, slots, v, vp), (k, v, slots, kp, k), (k, v, vp + 64, kp, vp), (kp, v, slots, kp, vp)):
        assert lib.lh_page_write(by, a[0], row, a[1], row, *a[2:], None) == -3, a
        assert "overlap" in lh.lh_last_error()
    assert lib.lh_page_write(by, k, 2 * row, v, row, slots, k + 2 * rows - 2 * row - 16, vp, None) == -3  # the last row's end
    need = lh.lh_paged_workspace_bytes(pc)
    q, table, cu, kv, o, lse, ws = M, 6 * M, 7 * M, 8 * M, 9 * M, 10 * M, 1 << 32
    good = [q, 8 * 64, kp, vp, table, cu, kv, o, lse, ws, need]
    for i, where in ((7, q), (7, kp + pool - 16), (7, vp), (7, table), (8, o + 100 * 8 * 64 * 2 - 4), (8, cu + 16), (9, o), (9, lse & -256),
                     (4, ws + 64), (6, lse), (0, ws + need - 256), (8, kv)):
        bad = list(good)
        bad[i] = where
        assert lib.lh_sdpa_paged(by, *bad, None) == -3 and "overlap" in lh.lh_last_error(), (i, hex(where))


class _Fake:
    """Stands in for a device tensor (only what the binding reads)."""

    def __init__(self, shape, dtype, stride=None, device=0):
        self.shape, self.dtype, self.is_cuda, self._device = tuple(shape), dtype, True, device
        dense, n = [], 1
        for x in reversed(self.shape):
            dense.insert(0, n)
            n *= x
        self._stride, self._n, self._dense = tuple(stride or dense), n, stride is None

    def numel(self):
        return self._n

    def stride(self):
        return self._stride

    def is_contiguous(self):
        return self._dense

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 0x1000


def _refused(call, args, i, bad, msg):
    args = list(args)
    args[i] = bad
    with pytest.raises(lh.LighthouseError, match=msg):
        call(*args)


def test_binding_refuses_bad_tensors():
    pc, i32, bf = _pc(), torch.int32, torch.bfloat16
    plan = [pc, _Fake([4], i32), _Fake([4], i32), _Fake([64], i32), _Fake([1], i32), _Fake([4, 8], i32), _Fake([5], i32),
            _Fake([4], i32), _Fake([100], i32), _Fake([100], i32), _Fake([1], i32)]
    for i, n in ((1, 4), (2, 4), (3, 64), (5, 32), (6, 5), (7, 4), (8, 100), (9, 100)):
        _refused(lh.lh_page_plan, plan, i, _Fake([n - 1], i32), "elements")
        _refused(lh.lh_page_plan, plan, i, _Fake([n], torch.int64), "dtype")
        _refused(lh.lh_page_plan, plan, i, _Fake([n], i32, device=1), "device 1")
    _refused(lh.lh_page_plan, plan, 5, _Fake([4, 8], i32, stride=(16, 1)), "not contiguous")
    _refused(lh.lh_page_plan, plan, 1, torch.zeros(4, dtype=i32), "not a device tensor")
    pool = _Fake([64, 2, 16, 64], bf)
    write = [pc, _Fake([100, 2, 64], bf), _Fake([100, 2, 64], bf), _Fake([100], i32), pool, pool]
    for i in (1, 2):
        _refused(lh.lh_page_write, write, i, _Fake([99, 2, 64], bf), "shape")
        _refused(lh.lh_page_write, write, i, _Fake([100, 128], bf), "shape")
        _refused(lh.lh_page_write, write, i, _Fake([100, 2, 64], bf, stride=(64, 6400, 1)), "within a token")
        _refused(lh.lh_page_write, write, i, _Fake([100, 2, 64], torch.float32), "dtype")
        _refused(lh.lh_page_write, write, i, _Fake([100, 2, 64], bf, device=3), "device 3")
    _refused(lh.lh_page_write, write, 4, _Fake([63, 2, 16, 64], bf), "elements")
    attend = [pc, _Fake([100, 8, 64], bf), pool, pool, _Fake([4, 8], i32), _Fake([5], i32), _Fake([4], i32),
              _Fake([100, 8, 64], bf), _Fake([100, 8], torch.float32), _Fake([1 << 30], torch.uint8)]
    for i, bad, msg in ((1, _Fake([100, 4, 64], bf), "shape"), (2, _Fake([64, 2, 16, 32], bf), "elements"),
                        (3, _Fake([64, 2, 16, 64], torch.float16), "dtype"), (4, _Fake([4, 7], i32), "elements"),
                        (5, _Fake([4], i32), "elements"), (6, _Fake([3], i32), "elements"),
                        (7, _Fake([99, 8, 64], bf), "elements"), (8, _Fake([100, 8], bf), "dtype"),
                        (9, _Fake([16], i32), "dtype"), (7, _Fake([100, 8, 64], bf, device=1), "device 1")):
        _refused(lh.lh_sdpa_paged, attend, i, bad, msg)


def test_binding_refuses_other_layouts():
    """As many elements in table rows of another width, or in pages laid out otherwise."""
    pc, i32, bf = _pc(), torch.int32, torch.bfloat16
    plan = [pc, _Fake([4], i32), _Fake([4], i32), _Fake([64], i32), _Fake([1], i32), _Fake([4, 8], i32), _Fake([5], i32),
            _Fake([4], i32), _Fake([100], i32), _Fake([100], i32), _Fake([1], i32)]
    pool = _Fake([64, 2, 16, 64], bf)
    write = [pc, _Fake([100, 2, 64], bf), _Fake([100, 2, 64], bf), _Fake([100], i32), pool, pool]
    attend = [pc, _Fake([100, 8, 64], bf), pool, pool, _Fake([4, 8], i32), _Fake([5], i32), _Fake([4], i32),
              _Fake([100, 8, 64], bf), _Fake([100, 8], torch.float32), _Fake([1 << 30], torch.uint8)]
    for call, args, at in ((lh.lh_page_plan, plan, 5), (lh.lh_sdpa_paged, attend, 4)):
        for shape in ([4, 9], [4, 16], [8, 4]):
            _refused(call, args, at, _Fake(shape, i32), "table has shape .* rows of")
    for call, args, ats in ((lh.lh_page_write, write, (4, 5)), (lh.lh_sdpa_paged, attend, (2, 3))):
        for at in ats:
            for shape in ([64, 16, 2, 64], [32, 2, 32, 64], [64, 4, 16, 64]):
                _refused(call, args, at, _Fake(shape, bf), "pages has shape .* rows of")


def test_binding_takes_layouts_that_are_the_same_memory():
    """A wider table of one request, pages of one head in another order, and one run of elements, are read as before."""
    i32, bf, need = torch.int32, torch.bfloat16, lh._need_laid
    for shape, dt, full in (([1, 9], i32, (1, 8)), ([4, 9], i32, (1, 8)), ([32], i32, (4, 8)), ([5, 8], i32, (4, 8)),
                            ([64, 16, 1, 64], bf, (64, 1, 16, 64)), ([32, 1, 32, 64], bf, (64, 1, 16, 64)),
                            ([65, 2, 16, 64], bf, (64, 2, 16, 64)), ([64 * 2 * 16 * 64], bf, (64, 2, 16, 64))):
        assert need("f", _Fake(shape, dt), "x", dt, full, 0) == 0x1000
    assert need("f", None, "x", i32, (1, 8), 0) is None and need("f", 4096, "x", i32, (1, 8), 0) == 4096


def test_reference_plan_hands_out_pages_in_order():
    """The oracle of the plan itself, on a case worked by hand: pages of 16; request 0 fills its page and takes one;
    request 1 brings nothing; request 2 lacks pages and waits; request 3 needs none and goes on; request 4 waits."""
    table = [[7, -1, -1], [3, -1, -1], [-1] * 3, [5, -1, -1], [-1] * 3]
    got = paged_ref.plan([10, 16, 0, 1, 0], [8, 0, 33, 2, 1], [20, 21, 22, 99], 3, table, 16, 64, 44)
    t, cu, kv, slots, pos, left, balance = got
    assert t == [[7, 22, -1], [3, -1, -1], [-1] * 3, [5, -1, -1], [-1] * 3]
    assert cu == [0, 8, 8, 41, 43, 44] and kv == [18, 16, 0, 3, 0] and left == 2 and balance == 3 - 4
    assert slots[:8] == [7 * 16 + x for x in range(10, 16)] + [22 * 16, 22 * 16 + 1]
    assert slots[8:41] == [-1] * 33 and slots[41:] == [81, 82, -1] and pos[41:] == [1, 2, -1]


def test_reference_attention_is_the_definition():
    """The oracle of the attention against a loop over keys, on pages in a mixed order, with an empty row."""
    g = torch.Generator().manual_seed(5)
    q = torch.randn(5, 2, 64, generator=g).to(torch.bfloat16)
    kp, vp = (torch.randn(6, 1, 16, 64, generator=g).to(torch.bfloat16) for _ in range(2))
    table, cu, kv = [[4, 1], [2, 0]], [0, 3, 5], [18, 1]
    o, lse, _, _ = paged_ref.attend(q, kp, vp, table, cu, kv, 16)
    for r, t, keys in ((0, 0, 16), (0, 2, 18), (1, 3, 0), (1, 4, 1)):
        for h in range(2):
            rows = [(table[r][j // 16], j % 16) for j in range(keys)]
            x = [float(q[t, h].double() @ kp[a, 0, b].double()) / 8 for a, b in rows]
            if not x:
                assert bool((o[t, h] == 0).all()) and float(lse[t, h]) == float("-inf")
                continue
            w = torch.tensor(x, dtype=torch.float64).softmax(0)
            ref = sum(p * vp[a, 0, b].double() for p, (a, b) in zip(w, rows))
            assert torch.allclose(o[t, h], ref, rtol=1e-12, atol=1e-14)
            assert abs(float(lse[t, h]) - float(torch.tensor(x, dtype=torch.float64).logsumexp(0))) < 1e-12
