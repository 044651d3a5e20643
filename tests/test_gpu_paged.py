"""Paged K/V cache operators on the GPU against the 64-bit reference."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests.helpers import cuda, i32

pytestmark = pytest.mark.gpu

S = pytest.importorskip("paper_2607_14557_gb300.seer")
TDT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    S.seer_check_device()
    yield
    torch.cuda.synchronize()


def rnd(rng, shape, dt, size=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * size).astype(np.float32)).to(TDT[dt]).to(cuda())


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound, what=""):
    """|got - ref| <= bound, NaN where ref is NaN."""
    got = host(got) if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - ref) <= bound + 1e-30)
    assert not bad.any(), (f"{what}: {int(bad.sum())}/{bad.size} outside the bound, first {np.argwhere(bad)[:4].tolist()}, "
                           f"got {got[bad][:4]}, want {ref[bad][:4]}, bound {np.broadcast_to(bound, got.shape)[bad][:4]}")


# ------------------------------------------------------------------ page tables
def run_tables(cached, new, page, free, head, table, n_pages, parents=None, mask=True, spare=3, stream=None):
    B, T = len(cached), sum(new)
    cap = T + spare
    t = dict(table=i32(table), cu=i32([-7] * (B + 1)), kv=i32([-7] * B), slot=i32([-7] * cap), pos=i32([-7] * cap),
             mask=torch.full((cap,), -7, dtype=torch.int64, device=cuda()) if mask else None, head=i32([-7]))
    par = i32([p for r in parents for p in r] + [0] * spare) if parents is not None else None
    S.seer_page_tables(i32(cached), i32(new), B, page, n_pages, i32(free), len(free), i32([head]), t["table"], len(table[0]), cap,
                       par, t["cu"], t["kv"], t["slot"], t["pos"], t["mask"], t["head"], stream=stream)
    return t


def make_tables(rng, cached, new, page, extra=5):
    """Random pages of the cached rows, a shuffled free list, the pool's size."""
    have = [math.ceil(c / page) for c in cached]
    most = max(math.ceil((c + n) / page) for c, n in zip(cached, new))
    need = sum(math.ceil((c + n) / page) for c, n in zip(cached, new))
    order = rng.permutation(need + extra)
    table, at = np.full((len(cached), max(most, 1) + 1), -5), 0
    for b, h in enumerate(have):
        table[b, :h] = order[at:at + h]
        at += h
    return table.tolist(), order[at:].tolist(), need + extra


def random_tree(rng, n):
    return [-1 if i == 0 else int(rng.integers(max(-1, i - 9), i)) for i in range(n)]


@pytest.mark.parametrize("B,cached,new,page", [(1, 1, 1, 16), (1, 0, 64, 8), (3, 40, 64, 16), (8, 4000, 1, 16), (33, 300, 20, 32),
                                               (257, 90, 64, 64), (700, 50, 9, 8), (5, 200, 64, 1024)])
@pytest.mark.parametrize("kind", ["tree", "chain", "nomask"])
def test_page_tables(B, cached, new, page, kind):
    rng = np.random.default_rng(B * 7 + page)
    c = [int(v) for v in rng.integers(0, cached + 1, B)]
    n = [int(v) for v in rng.integers(0, new + 1, B)]
    table, free, n_pages = make_tables(rng, c, n, page)
    parents = [random_tree(rng, m) for m in n] if kind == "tree" else None
    ref = R.page_tables(c, n, page, [0, 0] + free, 2, table, parents)
    for _ in range(2):                                  # a call may be repeated
        t = run_tables(c, n, page, [0, 0] + free, 2, table, n_pages, parents, mask=kind != "nomask")
        T = sum(n)
        assert t["cu"].tolist() == ref[0] and t["kv"].tolist() == ref[1]
        assert t["slot"].tolist() == ref[2] + [-7] * 3
        assert t["pos"].tolist() == ref[3] + [-7] * 3
        assert t["table"].tolist() == ref[5] and t["head"].tolist() == [ref[6]]
        if kind != "nomask":
            assert [v & (2 ** 64 - 1) for v in t["mask"].tolist()[:T]] == ref[4] and t["mask"].tolist()[T:] == [-7] * 3
    assert S.seer_check_device() == 0


def test_page_tables_long_prompts_and_large_batches():
    rng = np.random.default_rng(3)
    for B, hi, page in ((2, 20000, 64), (5000, 12, 16), (S.MAX_REQUESTS, 2, 8)):
        c = [int(v) for v in rng.integers(0, 40, B)]
        n = [int(v) for v in rng.integers(0, hi + 1, B)]
        table, free, n_pages = make_tables(rng, c, n, page)
        ref = R.page_tables(c, n, page, free, 0, table)
        t = run_tables(c, n, page, free, 0, table, n_pages, mask=False, spare=0)
        assert t["slot"].tolist() == ref[2] and t["table"].tolist() == ref[5] and t["cu"].tolist() == ref[0]
        assert t["pos"].tolist() == ref[3] and t["head"].tolist() == [ref[6]]
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("what,code", [("free list", 5), ("table", 5), ("rows", 1), ("negative", 2), ("page", 2), ("old page", 2),
                                       ("parent", 2), ("long draft", 2)])
def test_page_tables_record_what_does_not_fit(what, code):
    c, n, page = [10, 3], [20, 9], 8
    table, free, n_pages, parents, spare = [[0, 1, -1, -1], [2, -1, -1, -1]], [3, 4, 5, 6], 9, None, 0
    if what == "free list":
        free = free[:2]
    if what == "table":
        n = [30, 9]
    if what == "rows":
        spare = -4
    if what == "negative":
        c, n = [10, -3], [20, 0]
    if what == "page":
        free = [3, 900, 5, 6]
    if what == "old page":
        table[0][1] = 77
    if what == "parent":
        parents = [[-1, 1] + list(range(1, 19)), [-1] + list(range(8))]
    if what == "long draft":
        n, parents, free, table, n_pages = [70, 9], [[-1] * 70, [-1] * 9], list(range(3, 30)), [[0, 1] + [-1] * 12, [2] + [-1] * 13], 40
    t = run_tables(c, n, page, free, 0, table, n_pages, parents, mask=what in ("parent", "long draft"), spare=spare)
    assert S.seer_check_device() == code
    slot, tab = t["slot"].tolist(), t["table"].tolist()
    if what == "free list":         # the first request takes both pages, the second has none for its rows from 8 on
        assert tab == [[0, 1, 3, 4], [2, -1, -1, -1]] and slot[:20] == [10, 11, 12, 13, 14, 15] + list(range(24, 38))
        assert slot[20:] == [19, 20, 21, 22, 23] + [-1] * 4
    if what == "table":
        assert slot[22:30] == [-1] * 8 and t["kv"].tolist() == [32, 12] and tab[0] == [0, 1, 3, 4]
    if what == "rows":
        assert t["cu"].tolist() == [0, 20, 29]
    if what == "negative":
        assert t["cu"].tolist() == [0, 20, 20] and t["kv"].tolist() == [30, 0]
    if what == "page":
        assert tab[0] == [0, 1, 3, -1] and slot[14:20] == [-1] * 6
    if what == "old page":
        assert slot[:6] == [-1] * 6 and slot[6] == 24
    if what == "parent":            # row 1 names itself: it is a root
        assert t["mask"].tolist()[:3] == [1, 2, 6] and t["pos"].tolist()[:3] == [10, 10, 11]
    if what == "long draft":
        assert t["mask"].tolist()[:70] == [0] * 70 and t["mask"].tolist()[70:] == [1 << i for i in range(9)]


def test_page_tables_requests_of_nearly_2_31_rows():
    table = torch.zeros((1, 1 << 22), dtype=torch.int32, device=cuda())
    top = 2 ** 31 - 1025
    for c, n, code, kv, slot in [(top - 2, 2, 0, top, [1021, 1022]), (top - 1, 2, 5, top, [1022, -1]), (2 ** 31 - 1, 1, 5, top, [-1]),
                                 (2 ** 31 - 1, 2 ** 31 - 1, 5, top, [-1])]:
        out = [i32([-7] * 2), i32([-7]), i32([-7] * 2), i32([-7] * 2), i32([-7])]
        S.seer_page_tables(i32([c]), i32([n]), 1, 1024, 5, i32([3, 4]), 2, i32([0]), table, 1 << 22, min(n, 2), None, out[0], out[1], out[2],
                           out[3], None, out[4])
        got = S.seer_check_device()
        assert got == code or (code and got == 1)            # (more rows than slot_out holds is recorded too)
        assert out[1].tolist() == [kv] and out[4].tolist() == [0] and out[2].tolist()[:len(slot)] == slot


# ------------------------------------------------------------------ append
class Pool:
    """A pool of pages, a table of random pages for requests of kv rows each."""

    def __init__(self, rng, kv, page, hk, dh, dt, fill=1.0, extra=3):
        need = [math.ceil(v / page) for v in kv]
        self.n, self.page, self.hk, self.dh = sum(need) + extra, page, hk, dh
        self.max_pages = max(max(need), 1)
        order = rng.permutation(self.n)
        tab, at = np.full((len(kv), self.max_pages), -1), 0
        for b, m in enumerate(need):
            tab[b, :m] = order[at:at + m]
            at += m
        self.tab = tab.tolist()
        self.table = i32(tab)
        self.kv = rnd(rng, (self.n * page, 2 * hk * dh), dt, fill)
        self.struct = S.make_pages(self.kv, self.table, self.n, page, self.max_pages, hk, dh)

    def rows(self, b, t):
        return self.tab[b][t // self.page] * self.page + t % self.page


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hq,hk,dh,T,page", [(4, 2, 64, 1, 16), (32, 8, 128, 5, 64), (7, 1, 128, 37, 8), (6, 3, 16, 700, 128),
                                             (8, 8, 48, 64, 32), (4, 4, 128, 1300, 16)])
@pytest.mark.parametrize("mode", ["out", "inplace", "cache only", "no rotation"])
def test_append(dt, hq, hk, dh, T, page, mode):
    rng = np.random.default_rng(T + hq)
    pool = Pool(rng, [T + 9], page, hk, dh, dt)
    pad = 16
    x = rnd(rng, (T + 2, (hq + 2 * hk) * dh + pad), dt)
    pos = rng.integers(0, [60, 5000, 200000, 1 << 30][T % 4], T + 2)
    slot = np.array([pool.rows(0, t) for t in rng.permutation(T + 9)[:T + 2]])
    slot[rng.random(T + 2) < 0.1] = -1
    theta = 0.0 if mode == "no rotation" else 10000.0
    rot = {"inplace": x.clone(), "cache only": None}.get(mode, torch.full((T + 2, (hq + hk) * dh + 8 * 2), 3.0, dtype=TDT[dt], device=cuda()))
    src = rot if mode == "inplace" else x
    before_kv, before = host(pool.kv), host(rot) if rot is not None else None
    S.seer_kv_append(src, src.stride(0), dt, hq, T + 2, i32([T]), i32(slot), i32(pos) if theta else None, theta, rot,
                     rot.stride(0) if rot is not None else 0, pool.struct)
    xh = host(x)
    qk = xh[:T, :(hq + hk) * dh].reshape(T, hq + hk, dh)
    turned = R.rotate(qk, pos[:T], theta)
    bound = R.rotate_bound(qk, turned, dt) if theta else np.zeros_like(turned)
    if rot is not None:
        got = host(rot)
        close(got[:T, :(hq + hk) * dh], turned.reshape(T, -1), bound.reshape(T, -1), "rotated")
        assert (got[T:] == before[T:]).all() and (got[:T, (hq + hk) * dh:] == before[:T, (hq + hk) * dh:]).all()
    want, tol = before_kv.copy(), np.zeros_like(before_kv)
    for r in range(T):
        if slot[r] >= 0:
            want[slot[r]] = np.concatenate([turned[r, hq:].ravel(), xh[r, (hq + hk) * dh:(hq + 2 * hk) * dh]])
            tol[slot[r], :hk * dh] = bound[r, hq:].ravel()
    close(pool.kv, want, tol, "cache")
    assert S.seer_check_device() == 0


def test_append_records_slots_outside_the_pool_and_bad_row_counts():
    rng = np.random.default_rng(0)
    pool = Pool(rng, [40], 16, 2, 64, "bf16")
    x = rnd(rng, (4, 6 * 64), "bf16")
    before = pool.kv.clone()
    for bad in (pool.n * 16, 2 ** 31 - 1, -2, -2 ** 31):
        S.seer_kv_append(x, 384, "bf16", 2, 1, None, i32([bad]), None, 0.0, None, 0, pool.struct)
        assert S.seer_check_device() == 2 and torch.equal(before, pool.kv)
    S.seer_kv_append(x, 384, "bf16", 2, 2, i32([5]), i32([1, 2]), None, 0.0, None, 0, pool.struct)
    assert S.seer_check_device() == 1
    assert torch.equal(pool.kv[1], x[0, 128:]) and torch.equal(pool.kv[2], x[1, 128:])
    S.seer_kv_append(x, 384, "bf16", 2, 0, None, i32([1]), None, 0.0, None, 0, pool.struct)
    assert S.seer_check_device() == 0


def test_append_rows_with_one_slot_leave_pieces_of_either():
    rng = np.random.default_rng(1)
    pool = Pool(rng, [40], 16, 2, 64, "bf16")
    x = rnd(rng, (8, 6 * 64), "bf16")
    before = pool.kv.clone()
    S.seer_kv_append(x, 384, "bf16", 2, 8, None, i32([5] * 8), None, 0.0, None, 0, pool.struct)
    got, rows = pool.kv[5].reshape(-1, 8), x[:, 128:].reshape(8, -1, 8)
    assert (got == rows).all(-1).any(0).all()
    before[5] = pool.kv[5]
    assert torch.equal(before, pool.kv) and S.seer_check_device() == 0


# ------------------------------------------------------------------ accept
@pytest.mark.parametrize("dt,hk,dh,page", [("bf16", 8, 128, 16), ("f16", 1, 16, 8), ("f32", 3, 72, 64), ("f32", 8, 128, 128)])
def test_accept(dt, hk, dh, page):
    rng = np.random.default_rng(hk)
    cached = [0, 5, 130, 64, 1000, 77]
    draft = 64
    pool = Pool(rng, [c + draft for c in cached], page, hk, dh, dt)
    kept = [[], [0], list(range(64)), [63], sorted(rng.choice(64, 30, replace=False).tolist()), [0, 1, 2, 9, 10, 40]]
    acc = i32([k + [-1] * (draft - len(k)) for k in kept])
    want = host(pool.kv)
    for b, k in enumerate(kept):
        src = [want[pool.rows(b, cached[b] + a)].copy() for a in k]
        for i, row in enumerate(src):
            want[pool.rows(b, cached[b] + i)] = row
    out = i32([-1] * 6)
    S.seer_kv_accept(dt, i32(cached), acc, i32([len(k) for k in kept]), 6, draft, pool.struct, out)
    assert (host(pool.kv) == want).all() and out.tolist() == [c + len(k) for c, k in zip(cached, kept)]
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("cached,kept,n", [(5, [1, 1], 2), (5, [2, 1], 2), (5, [-1, 1], 2), (5, [0, 8], 2), (5, [0, 1], 9), (5, [0, 1], -1),
                                           (-1, [0, 1], 2), (43, [0, 6], 2), (2 ** 31 - 3, [0, 6], 2)])
def test_accept_keeps_nothing_of_a_bad_list(cached, kept, n):
    rng = np.random.default_rng(1)
    pool = Pool(rng, [48, 48], 16, 2, 64, "bf16")
    before = host(pool.kv)
    out = i32([-9, -9])
    S.seer_kv_accept("bf16", i32([cached, 3]), i32([kept + [-1] * 6, [2] + [-1] * 7]), i32([n, 1]), 2, 8, pool.struct, out)
    assert S.seer_check_device() == 2
    before[pool.rows(1, 3)] = before[pool.rows(1, 5)]
    assert (host(pool.kv) == before).all() and out.tolist() == [cached, 4]


# ------------------------------------------------------------------ causal attention
def causal_case(rng, lens, hq, hk, dh, dt, pad=0, spare=0, size=1.0):
    T = sum(lens)
    x = rnd(rng, (T + spare, (hq + 2 * hk) * dh + pad), dt, size)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
    return x, cu


def run_causal(x, cu, hq, hk, dh, dt, o=None, stream=None):
    cap, ld = x.shape[0], x.stride(0)
    o = torch.full((cap, hq * dh), 5.0, dtype=TDT[dt], device=cuda()) if o is None else o
    S.seer_attention_causal(x, ld, x[:, hq * dh:], ld, x[:, (hq + hk) * dh:], ld, o, o.stride(0), dt, i32(cu), len(cu) - 1, cap, hq, hk,
                            dh, stream=stream)
    return o


def causal_ref(x, cu, hq, hk, dh, dt):
    h = host(x)[:cu[-1], :(hq + 2 * hk) * dh].reshape(cu[-1], hq + 2 * hk, dh)
    return R.causal(h[:, :hq], h[:, hq:hq + hk], h[:, hq + hk:], cu, dt)


LENS = [[1], [2], [127], [128], [129], [1, 1, 1], [300], [64, 0, 65, 31], [513, 7], [1, 255, 256, 257], [1000]]
HEADS = [(1, 1), (4, 2), (8, 8), (8, 1), (7, 1), (6, 2), (5, 1)]


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("bf16", 64), ("f16", 128), ("f16", 64), ("f32", 64), ("f32", 128), ("f32", 36)])
@pytest.mark.parametrize("i", range(len(LENS)))
def test_causal(dt, dh, i):
    rng = np.random.default_rng(i)
    hq, hk = HEADS[(i + dh) % len(HEADS)]
    x, cu = causal_case(rng, LENS[i], hq, hk, dh, dt, pad=8 * (i % 3), spare=i % 4)
    o = run_causal(x, cu, hq, hk, dh, dt)
    ref, bound = causal_ref(x, cu, hq, hk, dh, dt)
    T = cu[-1]
    close(host(o)[:T].reshape(ref.shape), ref, bound, f"{LENS[i]} {hq}/{hk}")
    assert (host(o)[T:] == 5.0).all()                      # rows behind the last sequence
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("hq,hk", [(32, 8), (16, 16), (128, 1), (33, 3)])
def test_causal_many_heads(dt, dh, hq, hk):
    rng = np.random.default_rng(hq)
    x, cu = causal_case(rng, [33, 140, 5], hq, hk, dh, dt)
    ref, bound = causal_ref(x, cu, hq, hk, dh, dt)
    close(host(run_causal(x, cu, hq, hk, dh, dt)).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_causal_large_scores(dt):
    """Scores of some hundreds: the running maximum moves from tile to tile."""
    rng = np.random.default_rng(9)
    x, cu = causal_case(rng, [700], 4, 2, 128, dt, size=5.0)
    with torch.no_grad():                                   # later keys weigh more
        x[:, 4 * 128:6 * 128] *= torch.linspace(0.1, 1.5, 700, device=cuda())[:, None].to(x.dtype)
    ref, bound = causal_ref(x, cu, 4, 2, 128, dt)
    close(host(run_causal(x, cu, 4, 2, 128, dt)).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", [3, 130, 299])
def test_causal_rows_before_a_bad_one_do_not_see_it(dt, dh, bad, where):
    rng = np.random.default_rng(2)
    hq, hk = 4, 2
    x, cu = causal_case(rng, [40, 300, 20], hq, hk, dh, dt, spare=140)
    ref, bound = causal_ref(x, cu, hq, hk, dh, dt)
    x[40 + where, hq * dh:] = bad                           # its keys and values
    x[360:] = bad                                           # rows behind the last sequence
    got = host(run_causal(x, cu, hq, hk, dh, dt))[:360].reshape(ref.shape)
    fine = np.ones(360, bool)
    fine[40 + where:340] = False
    close(got[fine], ref[fine], bound[fine])
    if math.isnan(bad):
        assert np.isnan(got[~fine]).all()
    S.seer_check_device()


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f32", 64)])
def test_causal_infinite_values_reach_their_column_alone(dt, dh):
    rng = np.random.default_rng(4)
    x, cu = causal_case(rng, [200], 2, 1, dh, dt)
    ref, bound = causal_ref(x, cu, 2, 1, dh, dt)
    x[150, 3 * dh + 5] = math.inf
    got = host(run_causal(x, cu, 2, 1, dh, dt)).reshape(ref.shape)
    assert np.isposinf(got[150:, :, 5]).all()
    keep = np.ones(ref.shape, bool)
    keep[150:, :, 5] = False
    close(got[keep], ref[keep], bound[keep])
    S.seer_check_device()


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [300, 1400])
def test_causal_a_seen_nan_counts_whatever_its_weight(dt, dh, n):
    """Rows 3 and 257 score 0 where the keys from 130 on score dh * 25 / sqrt(dh) >= 200: e^-200 is 0 in 32 bits."""
    x = torch.zeros((n, 3 * dh), dtype=TDT[dt], device=cuda())
    x[:, :dh] = 5.0
    x[130:, dh:2 * dh] = 5.0
    x[257, dh:2 * dh] = 0.0
    x[:, 2 * dh:] = 1.0
    x[3, 2 * dh] = math.nan
    x[257, 2 * dh + 1] = math.nan
    o = host(run_causal(x, [0, n], 1, 1, dh, dt))
    want = np.ones((n, dh))
    want[3:, 0] = math.nan
    want[257:, 1] = math.nan
    assert np.array_equal(np.isnan(o), np.isnan(want))
    close(np.nan_to_num(o, nan=1.0), np.ones((n, dh)), 2.0 ** -7)
    S.seer_check_device()


def test_causal_separate_buffers_and_bad_offsets():
    rng = np.random.default_rng(5)
    dt, hq, hk, dh, lens = "bf16", 4, 2, 128, [100, 60]
    cu = [0, 100, 160]
    q, k, v = (rnd(rng, (170, h * dh + p), dt) for h, p in ((hq, 8), (hk, 64), (hk, 0)))
    o = torch.full((170, hq * dh + 24), 5.0, dtype=TDT[dt], device=cuda())

    def call(cu):
        S.seer_attention_causal(q, q.stride(0), k, k.stride(0), v, v.stride(0), o, o.stride(0), dt, i32(cu), 2, 170, hq, hk, dh)

    call(cu)
    assert S.seer_check_device() == 0
    heads = lambda t, h: host(t)[:160, :h * dh].reshape(160, h, dh)
    ref, bound = R.causal(heads(q, hq), heads(k, hk), heads(v, hk), cu, dt)
    close(heads(o, hq), ref, bound)
    assert (host(o)[:, hq * dh:] == 5.0).all() and (host(o)[160:] == 5.0).all()
    for bad in ([0, 100, 171], [-1, 100, 160], [0, 100, 90], [0, 2 ** 31 - 1, 160]):
        call(bad)
        assert S.seer_check_device() == 2, bad


# ------------------------------------------------------------------ attention of drafted rows
def run_tree(pool, q, cu, kv_len, hq, dt, mask=None, draft=None, spare=0, stream=None, ws=None, o=None):
    B = len(kv_len)
    draft = draft or max(max(np.diff(cu)), 1)
    size = S.seer_attention_tree_workspace_size(dt, B, hq, pool.hk, pool.dh, int(draft))
    ws = torch.full((size,), 255, dtype=torch.uint8, device=cuda()) if ws is None else ws
    o = torch.full((q.shape[0], hq * pool.dh), 5.0, dtype=TDT[dt], device=cuda()) if o is None else o
    words = None
    if mask is not None:
        words = torch.tensor([w - (1 << 64) if w >> 63 else w for w in mask] + [0] * (q.shape[0] - len(mask)), dtype=torch.int64, device=cuda())
    S.seer_attention_tree(q, q.stride(0), o, o.stride(0), dt, i32(cu), i32(kv_len), words, B, q.shape[0], hq, int(draft), pool.struct, ws,
                          ws.numel(), stream=stream)
    return o


def tree_ref(pool, q, cu, kv_len, hq, dt, mask=None):
    kv = host(pool.kv).reshape(-1, 2, pool.hk, pool.dh)
    qh = host(q)[:cu[-1], :hq * pool.dh].reshape(cu[-1], hq, pool.dh)
    return R.tree(qh, kv, pool.tab, pool.page, cu, kv_len, mask, dt)


def words_of(rng, new, kind):
    if kind == "causal":
        return None
    if kind == "all":
        return [(1 << n) - 1 for n in new for _ in range(n)]
    if kind == "none":
        return [0 for n in new for _ in range(n)]
    out = []
    for n in new:
        bits = []
        for i, p in enumerate(random_tree(rng, n)):
            bits.append((1 << i) | (bits[p] if p >= 0 else 0))
        out += bits
    return out


CTX = [([0], [1]), ([1], [1]), ([500], [1]), ([127, 128, 129], [1, 1, 1]), ([0, 300, 64], [64, 3, 17]), ([1000, 0, 0, 5], [2, 0, 5, 33]),
       ([2600], [64]), ([90, 4000], [8, 1])]


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("i", range(len(CTX)))
@pytest.mark.parametrize("kind", ["causal", "tree"])
def test_tree(dt, dh, i, kind):
    rng = np.random.default_rng(i + dh)
    ctx, new = CTX[i]
    hq, hk = HEADS[(i + dh // 64 + (kind == "tree")) % len(HEADS)]
    page = [8, 16, 32, 64, 128, 256][(i + dh // 64) % 6]
    kv_len = [c + n for c, n in zip(ctx, new)]
    pool = Pool(rng, kv_len, page, hk, dh, dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    q = rnd(rng, (cu[-1] + i % 3, hq * dh + 8 * (i % 2)), dt)
    mask = words_of(rng, new, kind)
    o = run_tree(pool, q, cu, kv_len, hq, dt, mask)
    ref, bound = tree_ref(pool, q, cu, kv_len, hq, dt, mask)
    close(host(o)[:cu[-1]].reshape(ref.shape), ref, bound, f"{ctx}+{new} {hq}/{hk} page {page}")
    assert (host(o)[cu[-1]:] == 5.0).all()
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("kind", ["all", "none"])
def test_tree_rows_that_see_all_or_nothing(dt, dh, kind):
    rng = np.random.default_rng(1)
    ctx, new, hq, hk = [0, 200, 0], [7, 30, 64], 4, 2
    kv_len = [c + n for c, n in zip(ctx, new)]
    pool = Pool(rng, kv_len, 16, hk, dh, dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    q = rnd(rng, (cu[-1], hq * dh), dt)
    mask = words_of(rng, new, kind)
    got = host(run_tree(pool, q, cu, kv_len, hq, dt, mask))
    ref, bound = tree_ref(pool, q, cu, kv_len, hq, dt, mask)
    close(got.reshape(ref.shape), ref, bound)
    if kind == "none":
        assert (got[:7] == 0).all() and (got[37:] == 0).all()
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("hq,hk,B", [(32, 8, 3), (64, 1, 2), (128, 1, 2), (16, 16, 1), (9, 3, 40)])
def test_tree_many_heads_and_requests(dt, dh, hq, hk, B):
    rng = np.random.default_rng(B)
    ctx = [int(v) for v in rng.integers(0, 900, B)]
    new = [int(v) for v in rng.integers(1, 9, B)]
    kv_len = [c + n for c, n in zip(ctx, new)]
    pool = Pool(rng, kv_len, 32, hk, dh, dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    q = rnd(rng, (cu[-1], hq * dh), dt)
    o = run_tree(pool, q, cu, kv_len, hq, dt, draft=8)
    ref, bound = tree_ref(pool, q, cu, kv_len, hq, dt)
    close(host(o).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_tree_hidden_and_stale_rows_do_not_count(dt, dh, bad):
    """Rows behind kv_len in a request's last page, and drafted rows that a row does not see."""
    rng = np.random.default_rng(6)
    hq, hk, ctx, new = 4, 2, [60, 250], [5, 9]
    kv_len = [65, 259]
    pool = Pool(rng, [c + 40 for c in kv_len], 32, hk, dh, dt)
    cu = [0, 5, 14]
    q = rnd(rng, (14, hq * dh), dt)
    mask = words_of(rng, new, "tree")
    hidden = 7                                              # drafted row 7 of request 1: seen by itself and its children
    ref, bound = tree_ref(pool, q, cu, kv_len, hq, dt, mask)
    used = {pool.rows(b, t) for b in range(2) for t in range(kv_len[b])}
    for r in range(pool.kv.shape[0]):
        if r not in used:
            pool.kv[r] = bad
    pool.kv[pool.rows(1, 250 + hidden)] = bad
    got = host(run_tree(pool, q, cu, kv_len, hq, dt, mask)).reshape(ref.shape)
    fine = np.array([True] * 5 + [not (w >> hidden) & 1 for w in mask[5:]])
    assert not fine.all()
    close(got[fine], ref[fine], bound[fine])
    S.seer_check_device()


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_tree_pages_outside_the_pool_read_as_zeros(dt, dh):
    rng = np.random.default_rng(7)
    hq, hk, kv_len, cu = 4, 2, [200, 90], [0, 2, 3]
    pool = Pool(rng, kv_len, 16, hk, dh, dt)
    q = rnd(rng, (3, hq * dh), dt)
    for bad in (-1, pool.n, 2 ** 31 - 1, -2 ** 31):
        tab = [list(r) for r in pool.tab]
        pool.table[0, 3] = bad
        o = run_tree(pool, q, cu, kv_len, hq, dt)
        assert S.seer_check_device() == 2
        kv = np.concatenate([host(pool.kv), np.zeros((16, 2 * hk * dh))]).reshape(-1, 2, hk, dh)
        tab[0][3] = pool.n
        ref, bound = R.tree(host(q).reshape(3, hq, dh), kv, tab, 16, cu, kv_len, None, dt)
        close(host(o).reshape(ref.shape), ref, bound)


def test_tree_records_lengths_that_do_not_fit():
    rng = np.random.default_rng(8)
    pool = Pool(rng, [64, 64], 16, 2, 128, "bf16")
    q = rnd(rng, (6, 4 * 128), "bf16")
    for cu, kv_len in (([0, 2, 4], [65, 64]), ([0, 2, 4], [1, 64]), ([0, 2, 7], [60, 64]), ([-1, 2, 4], [60, 64]), ([0, 4, 6], [60, 64]),
                       ([0, 2, 4], [-5, 64]), ([0, 2, 1], [60, 64]), ([0, 2, 4], [2 ** 31 - 1, 64]), ([0, 2, 4], [-2 ** 31, 64])):
        o = run_tree(pool, q, cu, kv_len, 4, "bf16", draft=3)
        assert S.seer_check_device() == 2, (cu, kv_len)
        if cu[2] == 4 and kv_len != [60, 64]:               # the other request's rows are there
            ref, bound = tree_ref(pool, q, cu, [2, 64], 4, "bf16")
            close(host(o)[2:4].reshape(2, 4, 128), ref[2:], bound[2:])
    with pytest.raises(S.SeerError, match="WORKSPACE"):
        S.seer_attention_tree(q, 512, torch.empty_like(q), 512, "bf16", i32([0, 2, 4]), i32([60, 64]), None, 2, 6, 4, 3, pool.struct, None, 0)


def test_tree_ignores_mask_bits_beyond_the_draft():
    rng = np.random.default_rng(21)
    for dt, dh in (("bf16", 128), ("f32", 64)):
        new, kv_len, cu = [3, 9], [130, 70], [0, 3, 12]
        pool = Pool(rng, kv_len, 16, 2, dh, dt)
        q = rnd(rng, (12, 4 * dh), dt)
        mask = words_of(rng, new, "tree")
        wide = [w | (((1 << 64) - 1) ^ ((1 << (3 if r < 3 else 9)) - 1)) for r, w in enumerate(mask)]
        a, b = run_tree(pool, q, cu, kv_len, 4, dt, mask), run_tree(pool, q, cu, kv_len, 4, dt, wide)
        assert torch.equal(a, b)
    assert S.seer_check_device() == 0


def test_pool_past_32_bit_offsets():
    """Pages behind the 4 GB and the 2^32-value mark of a pool."""
    rng = np.random.default_rng(22)
    dt, hq, hk, dh, page = "bf16", 8, 4, 128, 64
    n_pages = (1 << 33) // (page * 2 * hk * dh * 2) * 2 + 40          # 16 GB
    kv = torch.empty((n_pages * page, 2 * hk * dh), dtype=TDT[dt], device=cuda())
    ids = [n_pages - 1, 3, n_pages - 9, n_pages // 2, n_pages - 20, 0]
    table = i32([ids])
    pages = S.make_pages(kv, table, n_pages, page, len(ids), hk, dh)
    kv_len, T = 6 * 64 - 5, 20
    small = rnd(rng, (len(ids) * page, 2 * hk * dh), dt)
    for i, p in enumerate(ids):
        kv[p * page:(p + 1) * page] = small[i * page:(i + 1) * page]
    x = rnd(rng, (T, (hq + 2 * hk) * dh), dt)
    slot = [ids[t // page] * page + t % page for t in range(kv_len - T, kv_len)]
    S.seer_kv_append(x, x.stride(0), dt, hq, T, None, i32(slot), None, 0.0, None, 0, pages)
    small[kv_len - T:kv_len] = x[:, hq * dh:]
    for i, p in enumerate(ids):
        assert torch.equal(kv[p * page:(p + 1) * page], small[i * page:(i + 1) * page]), i
    size = S.seer_attention_tree_workspace_size(dt, 1, hq, hk, dh, T)
    ws = torch.empty(size, dtype=torch.uint8, device=cuda())
    o = torch.zeros((T, hq * dh), dtype=TDT[dt], device=cuda())
    S.seer_attention_tree(x, x.stride(0), o, o.stride(0), dt, i32([0, T]), i32([kv_len]), None, 1, T, hq, T, pages, ws, size)
    ref, bound = R.tree(host(x)[:, :hq * dh].reshape(T, hq, dh), host(small).reshape(-1, 2, hk, dh), [list(range(6))], page, [0, T],
                        [kv_len], None, dt)
    close(host(o).reshape(ref.shape), ref, bound)
    out = i32([0])
    S.seer_kv_accept(dt, i32([kv_len - T]), i32([[1, 5, 19] + [0] * 17]), i32([3]), 1, 20, pages, out)
    for k, a in enumerate((1, 5, 19)):
        assert torch.equal(kv[slot[k]], x[a, hq * dh:])
    assert S.seer_check_device() == 0 and out.tolist() == [kv_len - T + 3]


def test_causal_rows_past_32_bit_offsets():
    rng = np.random.default_rng(23)
    dt, hq, hk, dh, cap = "bf16", 4, 2, 128, 2_200_000
    w = (hq + 2 * hk) * dh                                            # 2.2e6 x 1024 values: past 2^31
    x = torch.empty((cap, w), dtype=TDT[dt], device=cuda())
    x[-300:] = rnd(rng, (300, w), dt)
    cu = [cap - 300, cap - 140, cap]
    o = torch.full((cap, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    run_causal(x, np.array(cu), hq, hk, dh, dt, o=o)
    ref, bound = causal_ref(x[-300:], np.array([0, 160, 300]), hq, hk, dh, dt)
    close(host(o[-300:]).reshape(ref.shape), ref, bound)
    assert (o[:-300] == 5.0).all()
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_causal_many_short_prompts(dt):
    rng = np.random.default_rng(24)
    lens = [int(v) for v in rng.integers(0, 5, 3000)]
    x, cu = causal_case(rng, lens, 4, 2, 64, dt)
    ref, bound = causal_ref(x, cu, 4, 2, 64, dt)
    close(host(run_causal(x, cu, 4, 2, 64, dt)).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("hq,hk,dh", [(32, 8, 128), (8, 8, 64), (16, 2, 128)])
def test_causal_many_units_per_sm(hq, hk, dh):
    """Dozens of short units in a row on every SM, after a few long ones."""
    rng = np.random.default_rng(27)
    lens = [700] + [int(v) for v in rng.integers(1, 200, 150)] + [400]
    x, cu = causal_case(rng, lens, hq, hk, dh, "bf16")
    ref, bound = causal_ref(x, cu, hq, hk, dh, "bf16")
    close(host(run_causal(x, cu, hq, hk, dh, "bf16")).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_tree_many_requests(dt):
    rng = np.random.default_rng(25)
    B = 1500
    new = [int(v) for v in rng.integers(0, 3, B)]
    kv_len = [int(v) + n for v, n in zip(rng.integers(0, 70, B), new)]
    pool = Pool(rng, kv_len, 8, 1, 64, dt)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    q = rnd(rng, (cu[-1], 3 * 64), dt)
    ref, bound = tree_ref(pool, q, cu, kv_len, 3, dt)
    close(host(run_tree(pool, q, cu, kv_len, 3, dt)).reshape(ref.shape), ref, bound)
    assert S.seer_check_device() == 0


def test_streams_given_and_launch_overlap_off():
    rng = np.random.default_rng(26)
    dt, hq, hk, dh = "f16", 4, 2, 128
    x, cu = causal_case(rng, [200, 90], hq, hk, dh, dt)
    pool = Pool(rng, [300, 64], 16, hk, dh, dt)
    q = rnd(rng, (7, hq * dh), dt)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = run_causal(x, cu, hq, hk, dh, dt), run_tree(pool, q, [0, 3, 7], [300, 64], hq, dt)
    torch.cuda.synchronize()
    outs = []
    before = S.seer_set_launch_overlap(False)
    try:
        for s in (side, side.cuda_stream, None):
            a = torch.full_like(want[0], 5.0)
            b = torch.full_like(want[1], 5.0)
            torch.cuda.synchronize()
            outs.append((run_causal(x, cu, hq, hk, dh, dt, o=a, stream=s), run_tree(pool, q, [0, 3, 7], [300, 64], hq, dt, o=b, stream=s)))
            torch.cuda.synchronize()
    finally:
        S.seer_set_launch_overlap(before)
    for a, b in outs:
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    assert S.seer_check_device() == 0


# ------------------------------------------------------------------ together
def test_prompt_draft_accept_steps():
    """Prompts, then rounds of drafting a tree, attending, and keeping a path of it: every
    output against dense attention over the tokens that each row descends from."""
    rng = np.random.default_rng(11)
    dt, hq, hk, dh, page, theta = "f32", 4, 2, 64, 16, 10000.0
    w, B, n_pages, max_pages = (hq + 2 * hk) * dh, 3, 60, 16
    kv = torch.full((n_pages * page, 2 * hk * dh), math.nan, device=cuda())
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device=cuda())
    pages = S.make_pages(kv, table, n_pages, page, max_pages, hk, dh)
    free = i32(rng.permutation(n_pages))
    head, cached = i32([0]), i32([0] * B)
    past = [[] for _ in range(B)]                          # unrotated (k, v) rows kept so far

    def layout(new, parents):
        cap = sum(new) + 2
        out = [torch.zeros(s, dtype=torch.int32, device=cuda()) for s in (B + 1, B, cap, cap)]
        mask = torch.zeros(cap, dtype=torch.int64, device=cuda()) if parents else None
        head_out = torch.zeros(1, dtype=torch.int32, device=cuda())
        par = i32([p for r in parents for p in r] + [0, 0]) if parents else None
        S.seer_page_tables(cached, i32(new), B, page, n_pages, free, n_pages, head, table, max_pages, cap, par, *out, mask, head_out)
        return *out, mask, head_out, cap

    def check(o, x, cu, ancestors, tag):
        for b in range(B):
            for i in range(cu[b + 1] - cu[b]):
                rows = past[b] + [(x[cu[b] + j, hq:hq + hk], x[cu[b] + j, hq + hk:]) for j in ancestors[b][i]]
                k = R.rotate(np.stack([r[0] for r in rows]), range(len(rows)), theta)
                v = np.stack([r[1] for r in rows])
                q = R.rotate(x[cu[b] + i, :hq][None], [len(rows) - 1], theta)[0]
                for h in range(hq):
                    ref, bound = R.attend(q[h][None], k[:, h // 2], v[:, h // 2], np.ones((1, len(rows)), bool), dt)
                    # the rotated rows carry fp32 roundings of their own into scores of size up to ~|q||k|
                    close(o[cu[b] + i, h][None], ref, bound + 1e-5, f"{tag} {b}.{i}")

    new = [30, 1, 47]
    cu, kv_len, slot, pos, _, head_out, cap = layout(new, None)
    x = rnd(rng, (cap, w), dt)
    xh = host(x).reshape(cap, -1, dh)
    S.seer_kv_append(x, w, dt, hq, cap, cu[B:], slot, pos, theta, x, w, pages)
    o = torch.zeros((cap, hq * dh), device=cuda())
    S.seer_attention_causal(x, w, x[:, hq * dh:], w, x[:, (hq + hk) * dh:], w, o, hq * dh, dt, cu, B, cap, hq, hk, dh)
    c = cu.tolist()
    check(host(o).reshape(cap, hq, dh), xh, c, [[list(range(i + 1)) for i in range(n)] for n in new], "prompt")
    for b in range(B):
        past[b] += [(xh[r, hq:hq + hk], xh[r, hq + hk:]) for r in range(c[b], c[b + 1])]
    head.copy_(head_out)
    cached.copy_(kv_len)
    for step in range(4):
        new = [int(v) for v in rng.integers(1, 20, B)]
        parents = [random_tree(rng, n) for n in new]
        lines = []
        for pr in parents:
            anc = []
            for i, p in enumerate(pr):
                anc.append((anc[p] if p >= 0 else []) + [i])
            lines.append(anc)
        cu, kv_len, slot, pos, mask, head_out, cap = layout(new, parents)
        x = rnd(rng, (cap, w), dt)
        xh = host(x).reshape(cap, -1, dh)
        S.seer_kv_append(x, w, dt, hq, cap, cu[B:], slot, pos, theta, x, w, pages)
        size = S.seer_attention_tree_workspace_size(dt, B, hq, hk, dh, 20)
        ws = torch.empty(size, dtype=torch.uint8, device=cuda())
        o = torch.zeros((cap, hq * dh), device=cuda())
        S.seer_attention_tree(x, w, o, hq * dh, dt, cu, kv_len, mask, B, cap, hq, 20, pages, ws, size)
        c = cu.tolist()
        check(host(o).reshape(cap, hq, dh), xh, c, lines, f"step {step}")
        kept = [ln[int(rng.integers(0, len(ln)))] for ln in lines]
        S.seer_kv_accept(dt, cached, i32([k + [-1] * (20 - len(k)) for k in kept]), i32([len(k) for k in kept]), B, 20, pages, kv_len)
        for b in range(B):
            past[b] += [(xh[c[b] + r, hq:hq + hk], xh[c[b] + r, hq + hk:]) for r in kept[b]]
        # pages that only rejected rows filled stay in the table: the next step finds them there
        cached.copy_(kv_len)
        assert cached.tolist() == [len(r) for r in past]
        head.copy_(head_out)
    assert S.seer_check_device() == 0


def test_captured_step_replays_on_new_lengths():
    """Tables, append and attention in one graph: lengths and rows are read at replay."""
    rng = np.random.default_rng(12)
    dt, hq, hk, dh, page, B, n_pages, max_pages, cap = "bf16", 8, 2, 128, 16, 4, 300, 40, 40
    w = (hq + 2 * hk) * dh
    kv = rnd(rng, (n_pages * page, 2 * hk * dh), dt)
    free, head, head_out = i32(rng.permutation(n_pages)), i32([0]), i32([0])
    table = i32(np.full((B, max_pages), -1))
    pages = S.make_pages(kv, table, n_pages, page, max_pages, hk, dh)
    cached, new = i32([0] * B), i32([1] * B)
    cu, kv_len, slot, pos = i32([0] * (B + 1)), i32([0] * B), i32([0] * cap), i32([0] * cap)
    x, rot = rnd(rng, (cap, w), dt), torch.zeros((cap, (hq + hk) * dh), dtype=TDT[dt], device=cuda())
    o = torch.zeros((cap, hq * dh), dtype=TDT[dt], device=cuda())
    size = S.seer_attention_tree_workspace_size(dt, B, hq, hk, dh, 10)
    ws = torch.empty(size, dtype=torch.uint8, device=cuda())

    def step():
        S.seer_page_tables(cached, new, B, page, n_pages, free, n_pages, head, table, max_pages, cap, None, cu, kv_len, slot, pos, None, head_out)
        S.seer_kv_append(x, w, dt, hq, cap, cu[B:], slot, pos, 10000.0, rot, rot.stride(0), pages)
        S.seer_attention_tree(rot, rot.stride(0), o, o.stride(0), dt, cu, kv_len, None, B, cap, hq, 10, pages, ws, size)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for trial in range(3):
        c = [int(v) for v in rng.integers(0, 600, B)]
        n = [int(v) for v in rng.integers(0, 11, B)]
        tab, fr, _ = make_tables(rng, c, n, page, extra=0)
        full = np.full((B, max_pages), -1)
        full[:, :len(tab[0])] = np.array(tab)[:, :max_pages]
        spare = [p for p in range(n_pages) if p not in {v for r in tab for v in r} and p not in fr]
        cached.copy_(i32(c))
        new.copy_(i32(n))
        table.copy_(i32(full))
        free.copy_(i32((fr + spare + [0] * n_pages)[:n_pages]))
        x.copy_(rnd(rng, (cap, w), dt))
        o.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        cl = cu.tolist()
        assert cl == [0] + np.cumsum(n).tolist() and kv_len.tolist() == [a + b for a, b in zip(c, n)]
        q = host(rot)[:cl[-1], :hq * dh].reshape(-1, hq, dh)
        ref, bound = R.tree(q, host(kv).reshape(-1, 2, hk, dh), table.tolist(), page, cl, kv_len.tolist(), None, dt)
        close(host(o)[:cl[-1]].reshape(ref.shape), ref, bound, f"replay {trial}")
        assert (host(o)[cl[-1]:] == 5.0).all()
    assert S.seer_check_device() == 0


def test_two_streams_at_once():
    rng = np.random.default_rng(13)
    dt, hq, hk, dh = "bf16", 8, 2, 128
    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = []
    for s, lens in zip(streams, ([700, 90], [33, 900])):
        x, cu = causal_case(rng, lens, hq, hk, dh, dt)
        pool = Pool(rng, [v + 5 for v in lens], 16, hk, dh, dt)
        q = rnd(rng, (10, hq * dh), dt)
        jobs.append((s, x, cu, pool, q, [v + 5 for v in lens]))
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        for s, x, cu, pool, q, kv_len in jobs:
            with torch.cuda.stream(s):
                outs.append((run_causal(x, cu, hq, hk, dh, dt), run_tree(pool, q, [0, 5, 10], kv_len, hq, dt)))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(outs):
        _, x, cu, pool, q, kv_len = jobs[i % 2]
        if i < 2:
            ref, bound = causal_ref(x, cu, hq, hk, dh, dt)
            close(host(a).reshape(ref.shape), ref, bound)
            ref, bound = tree_ref(pool, q, [0, 5, 10], kv_len, hq, dt)
            close(host(b).reshape(ref.shape), ref, bound)
        assert torch.equal(a, outs[i % 2][0]) and torch.equal(b, outs[i % 2][1])
    assert S.seer_check_device() == 0


def test_binding_refuses_tensors_elsewhere():
    x = torch.zeros((4, 512), dtype=torch.bfloat16)
    g = x.to(cuda())
    with pytest.raises(ValueError, match="current device"):
        S.seer_attention_causal(x, 512, g, 512, g, 512, g.clone(), 512, "bf16", i32([0, 4]), 1, 4, 2, 1, 128)
    pool = Pool(np.random.default_rng(0), [40], 16, 2, 128, "bf16")
    with pytest.raises(ValueError, match="range"):          # a workspace of -1 bytes is not a large one
        S.seer_attention_tree(g, 512, g.clone(), 512, "bf16", i32([0, 4]), i32([40]), None, 1, 4, 4, 4, pool.struct, g, -1)
    with pytest.raises(ValueError, match="Int"):
        S.seer_attention_causal(g, 512, g[:, 256:], 512, g[:, 384:], 512, g.clone(), 512, "bf16", i32([0, 4]).long(), 1, 4, 2, 1, 128)
