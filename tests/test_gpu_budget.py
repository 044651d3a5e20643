"""Rotary positions, attention mass, the choice of rows and their moves on the GPU against the 64-bit
reference, and a run of them as a server makes it."""
import math

import numpy as np
import pytest
import torch

from tests import budget_reference as R
from tests import paged_reference as PR
from tests.helpers import cuda, i32

pytestmark = pytest.mark.gpu

S = pytest.importorskip("paper_2607_14557_gb300.seer")
TDT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SCALES = {"none": {}, "linear": dict(factor=4.0), "turns": dict(factor=8.0, low=1.0, high=4.0, length=8192),
          "pairs": dict(factor=16.0, low=1.0, high=32.0, length=4096)}


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
    """|got - ref| <= bound, NaN exactly where ref is NaN."""
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert (np.isnan(got) == np.isnan(ref)).all(), f"{what}: NaN at {np.argwhere(np.isnan(got) != np.isnan(ref))[:4].tolist()}"
    bad = ~(np.abs(got - ref) <= bound + 1e-30) & ~np.isnan(ref)
    assert not bad.any(), (f"{what}: {int(bad.sum())}/{bad.size} outside the bound, first {np.argwhere(bad)[:4].tolist()}, "
                           f"got {got[bad][:4]}, want {ref[bad][:4]}, bound {np.broadcast_to(bound, got.shape)[bad][:4]}")


def rotary(theta, rd, inter, scaling, magnitude=1.0):
    kw = dict(SCALES[scaling])
    length = kw.pop("length", 1)
    return (S.make_rotary(theta, rd, interleaved=inter, scaling=scaling, original_len=length, magnitude=magnitude, **kw),
            R.rates(theta, rd, scaling, length=length, **kw))


# ------------------------------------------------------------------ rotated rows
@pytest.mark.parametrize("dt,heads,dh,rd", [("bf16", 5, 128, 128), ("bf16", 3, 128, 32), ("f16", 2, 64, 4), ("f16", 7, 80, 20),
                                            ("bf16", 1, 96, 72), ("f32", 3, 80, 20), ("f32", 2, 8, 2), ("f32", 4, 128, 124),
                                            ("f32", 1, 40, 36), ("bf16", 2, 112, 112)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rows", [1, 37, 1300])
def test_rotate(dt, heads, dh, rd, inter, rows):
    rng = np.random.default_rng(heads * 100 + rd + rows)
    pad, spare = 16, 2
    scaling = list(SCALES)[(rows + rd) % 4]
    rot, rate = rotary(10000.0, rd, inter, scaling, 1.25 if scaling == "pairs" else 1.0)
    magnitude = rot.magnitude
    x = rnd(rng, (rows + spare, heads * dh + pad), dt)
    pos = np.concatenate([rng.integers(0, 200000, rows - 1), [2 ** 31 - 1 if rows > 1 else 7]])
    if rows > 4:
        pos[:3] = [0, 1, -5]
    ref = R.turn(host(x[:rows, :heads * dh]).reshape(rows, heads, dh), pos, rate, inter, magnitude)
    bound = R.turn_bound(host(x[:rows, :heads * dh]).reshape(rows, heads, dh), ref, pos, rd, inter, dt, magnitude)
    out = torch.full((rows + spare, heads * dh + 8), 5.0, dtype=TDT[dt], device=cuda())
    before = x.clone()
    position = i32(list(pos) + [9] * spare)
    S.seer_rotate(x, x.stride(0), dt, heads, dh, rows + spare, i32([rows]), position, rot, out, out.stride(0))
    assert torch.equal(x, before)
    close(out[:rows, :heads * dh].reshape(rows, heads, dh), ref, bound, "out")
    assert (out[rows:] == 5).all() and (out[:, heads * dh:] == 5).all()
    S.seer_rotate(x, x.stride(0), dt, heads, dh, rows, None, position, rot, x, x.stride(0))
    assert torch.equal(x[:rows, :heads * dh], out[:rows, :heads * dh])
    assert torch.equal(x[rows:], before[rows:]) and torch.equal(x[:, heads * dh:], before[:, heads * dh:])
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("inter", [False, True])
def test_rotate_leaves_infinities_of_the_plain_part_and_other_pairs_alone(inter):
    rot, _ = rotary(10000.0, 12, inter, "none")
    x = torch.ones(3, 32, device=cuda())
    x[:, 12:] = math.inf
    x[1, 0], x[2, 31] = math.nan, math.nan
    out = torch.zeros_like(x)
    S.seer_rotate(x, 32, "f32", 1, 32, 3, None, i32([3, 4, 5]), rot, out, 32)
    assert torch.equal(out[:, 12:31], x[:, 12:31]) and out[2, 31].isnan()
    bad = {0, 1 if inter else 6}
    assert {i for i in range(12) if out[1, i].isnan()} == bad and not out[0].isnan().any() and not out[2, :31].isnan().any()


def test_rotate_records_a_bad_row_count():
    rot, _ = rotary(100.0, 16, False, "none")
    x = torch.ones(4, 16, device=cuda())
    S.seer_rotate(x, 16, "f32", 1, 16, 4, i32([9]), i32([0] * 4), rot, x, 16)
    assert S.seer_check_device() == 1 and (x == 1).all()
    S.seer_rotate(x, 16, "f32", 1, 16, 4, i32([-2]), i32([1] * 4), rot, x, 16)
    assert S.seer_check_device() == 1 and (x == 1).all()


# ------------------------------------------------------------------ rotated rows into the cache
@pytest.mark.parametrize("dt,hq,hk,dh,rd,inter,scaling", [
    ("bf16", 8, 2, 128, 128, True, "turns"), ("f16", 4, 4, 64, 16, False, "pairs"), ("f32", 3, 1, 40, 36, False, "linear"),
    ("f32", 2, 2, 8, 6, True, "none"), ("bf16", 6, 3, 80, 20, False, "turns"), ("bf16", 2, 1, 16, None, False, "none")])
@pytest.mark.parametrize("new", [[1, 0, 3, 1], [40] * 40])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_rotary(dt, hq, hk, dh, rd, inter, scaling, new, in_place):
    rng = np.random.default_rng(dh + len(new))
    B, T, spare, page = len(new), sum(new), 3, 8
    rot, rate = rotary(500000.0, rd, inter, scaling) if rd else (None, [])
    width = (hq + 2 * hk) * dh
    x = rnd(rng, (T + spare, width + 8), dt)
    before = x.clone()
    pos = rng.integers(0, 5000, T + spare)
    shift = rng.integers(0, 90000, B)
    owner = np.concatenate([np.repeat(np.arange(B), new), [-1] * spare]).astype(int)
    moved = [int(p) + (int(shift[b]) if b >= 0 else 0) for p, b in zip(pos, owner)]
    pool_rows = (T // page + 3) * page
    slot = rng.permutation(pool_rows)[:T + spare]
    slot[[0, -1]] = -1
    kv = rnd(rng, (pool_rows, 2 * hk * dh), dt)
    kv0 = kv.clone()
    table = i32([[0]])
    pages = S.make_pages(kv, table, pool_rows // page, page, 1, hk, dh)
    rotated = x if in_place else torch.full((T + spare, (hq + hk) * dh + 16), 5.0, dtype=TDT[dt], device=cuda())
    S.seer_kv_append_rotary(x, x.stride(0), dt, hq, T + spare, None, i32(slot), i32(pos), i32(np.concatenate([[0], np.cumsum(new)])),
                            i32(shift), B, rot, rotated, rotated.stride(0), pages)
    heads = host(before[:, :width]).reshape(T + spare, hq + 2 * hk, dh)
    ref = R.turn(heads[:, :hq + hk], moved, rate, inter)
    bound = R.turn_bound(heads[:, :hq + hk], ref, moved, 2 * len(rate), inter, dt)
    close(rotated[:, :(hq + hk) * dh].reshape(T + spare, hq + hk, dh), ref, bound, "rotated")
    if in_place:
        assert torch.equal(x[:, (hq + hk) * dh:], before[:, (hq + hk) * dh:])
    else:
        assert torch.equal(x, before) and (rotated[:, (hq + hk) * dh:] == 5).all()
    there = slot >= 0
    got = kv[torch.from_numpy(slot[there]).to(cuda())].reshape(-1, 2, hk, dh)
    assert torch.equal(got[:, 0].reshape(-1, hk * dh), rotated[torch.from_numpy(there).to(cuda()), hq * dh:(hq + hk) * dh])
    assert torch.equal(got[:, 1].reshape(-1, hk * dh), before[torch.from_numpy(there).to(cuda()), (hq + hk) * dh:width])
    rest = np.setdiff1d(np.arange(pool_rows), slot[there])
    assert torch.equal(kv[torch.from_numpy(rest).to(cuda())], kv0[torch.from_numpy(rest).to(cuda())])
    assert S.seer_check_device() == 0


def test_append_rotary_without_shift_is_append():
    rng = np.random.default_rng(3)
    hq, hk, dh, T = 4, 2, 128, 50
    x = rnd(rng, (T, (hq + 2 * hk) * dh), "bf16")
    outs = []
    rot, _ = rotary(10000.0, dh, False, "none")
    pos, slot = i32(rng.integers(0, 8000, T)), i32(rng.permutation(64)[:T])
    for own in (False, True):
        kv, out = torch.zeros(64, 2 * hk * dh, dtype=torch.bfloat16, device=cuda()), torch.zeros(T, (hq + hk) * dh, dtype=torch.bfloat16, device=cuda())
        table = i32([[0]])
        pages = S.make_pages(kv, table, 8, 8, 1, hk, dh)
        if own:
            S.seer_kv_append_rotary(x, x.stride(0), "bf16", hq, T, None, slot, pos, None, None, 0, rot, out, out.stride(0), pages)
        else:
            S.seer_kv_append(x, x.stride(0), "bf16", hq, T, None, slot, pos, 10000.0, out, out.stride(0), pages)
        outs.append((kv, out))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B", [1, 31, 33, 1024, 1025, 5000])
def test_append_rotary_finds_the_request_of_a_row(B):
    # rows of 0 .. 3 a request: by heads of one pair that turns a quarter per position
    rng = np.random.default_rng(B)
    new = rng.integers(0, 4, B)
    new[-1] = 1
    T = int(new.sum())
    rot = S.make_rotary(1.0, 2, interleaved=True)
    x = torch.zeros(T, 24, device=cuda())
    x[:, 0] = 1
    shift = rng.integers(0, 1000, B)
    kv, table = torch.zeros(8, 16, device=cuda()), i32([[0]])
    S.seer_kv_append_rotary(x, 24, "f32", 1, T, None, i32([-1] * T), i32([0] * T), i32(np.concatenate([[0], np.cumsum(new)])), i32(shift), B,
                            rot, x, 24, S.make_pages(kv, table, 1, 8, 1, 1, 8))
    angle = np.repeat(shift, new).astype(float)
    close(x[:, 0], np.cos(angle), 2.0 ** -20, "cos")
    close(x[:, 1], np.sin(angle), 2.0 ** -20, "sin")


# ------------------------------------------------------------------ attention mass
def setup_mass(rng, dt, hq, hk, dh, page, cached, new, accepted=None, pad=0, spare_ld=5, size=1.0):
    """Pool, table and queries; accepted: per request the accepted rows of its draft."""
    left = [len(a) for a in accepted] if accepted else new
    kv_len = [c + n for c, n in zip(cached, left)]
    need = [math.ceil(t / page) for t in kv_len]
    n_pages, max_pages = sum(need) + 3, max(max(need), 1) + 1
    order = rng.permutation(n_pages)
    table, at = np.full((len(cached), max_pages), -1), 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    kv = rnd(rng, (n_pages * page, 2 * hk * dh), dt)
    q = rnd(rng, (sum(new) + 2, hq * dh + pad), dt, size)
    return dict(kv=kv, table=table, q=q, kv_len=kv_len, cu=np.concatenate([[0], np.cumsum(new)]), n_pages=n_pages, max_pages=max_pages,
                ld=max(max(kv_len), 1) + spare_ld)


def run_mass(s, dt, hq, hk, dh, page, window, keep, mass_in, gone, accepted=None, in_place=False, T_kv_cap=None, draft=None, ws_fill=255, stream=None):
    B = len(s["kv_len"])
    table = i32(s["table"])                      # the struct keeps its address only
    pages = S.make_pages(s["kv"], table, s["n_pages"], page, s["max_pages"], hk, dh)
    cap = sum(s["kv_len"]) if T_kv_cap is None else T_kv_cap
    ws_bytes = S.seer_attention_mass_workspace_size(dt, B, cap, hq, hk, dh, window)
    ws = torch.full((ws_bytes,), ws_fill, dtype=torch.uint8, device=cuda())
    acc = n_acc = None
    draft = draft or max([1] + [len(a) for a in accepted] if accepted else [1])
    if accepted:
        acc, n_acc = i32([list(a) + [-1] * (draft - len(a)) for a in accepted]), i32([len(a) for a in accepted])
    out = mass_in.clone() if in_place else torch.full_like(mass_in, -3.0)
    birth = torch.full(mass_in.shape, -9, dtype=torch.int32, device=cuda())
    S.seer_attention_mass(s["q"], s["q"].stride(0), dt, i32(s["cu"]), i32(s["kv_len"]), acc, n_acc, draft, window, B, s["q"].shape[0], cap, hq,
                          pages, keep, None if gone is None else i32(gone), (out if in_place else mass_in) if keep else None, out, birth, s["ld"],
                          ws, ws_bytes, stream=stream)
    return out, birth


def check_mass(s, out, birth, dt, hq, hk, dh, page, window, keep, mass_in, gone, accepted=None, untouched=-3.0):
    B = len(s["kv_len"])
    q = host(s["q"])[:, :hq * dh].reshape(-1, hq, dh)
    keys = host(s["kv"])[:, :hk * dh].reshape(-1, hk, dh)
    requests = []
    for b, kv in enumerate(s["kv_len"]):
        n = len(accepted[b]) if accepted else int(s["cu"][b + 1] - s["cu"][b])
        places = list(range(max(0, n - window), n))
        requests.append(([int(s["cu"][b]) + (accepted[b][i] if accepted else i) for i in places], places, n, kv))
    ref = R.mass(q, keys, s["table"], page, requests, keep, host(mass_in), dh)
    old = host(mass_in)
    for b in range(B):
        kv, n = s["kv_len"][b], requests[b][2]
        close(out[b, :kv], ref[b][0], ref[b][1], f"request {b}")
        after = host(out[b, kv:])
        assert (after == (old[b, kv:] if untouched is None else untouched)).all()
        want = np.full(s["ld"], -9)
        want[kv - n:kv] = np.arange(kv - n, kv) + (gone[b] if gone is not None else 0)
        assert (birth[b].cpu().numpy() == want).all()


MASS = [  # dt, hq, hk, dh, page, cached, new, window
    ("bf16", 8, 2, 128, 16, [700, 433, 0, 1], [1, 1, 1, 1], 1),
    ("f16", 32, 8, 128, 64, [5, 63, 64, 65, 127, 128, 129], [1] * 7, 1),
    ("bf16", 4, 4, 64, 8, [90, 0, 33], [3, 9, 0], 4),
    ("f16", 6, 2, 64, 16, [200, 0, 0, 17], [5, 1, 64, 2], 64),
    ("bf16", 16, 2, 128, 32, [0, 300], [77, 40], 33),
    ("bf16", 7, 1, 128, 16, [1000], [2], 2),
    ("f16", 5, 5, 128, 16, [31, 64, 100], [1, 1, 2], 2),
    ("bf16", 24, 3, 64, 8, [70, 129], [1, 1], 1),
    ("f32", 4, 2, 64, 8, [1, 17, 130, 255], [24, 1, 3, 0], 24),
    ("f32", 3, 1, 40, 16, [900], [1], 1),
    ("f32", 2, 2, 128, 1024, [1500, 0], [9, 64], 64),
    ("bf16", 128, 1, 64, 16, [129], [2], 2),
    ("f16", 36, 4, 128, 16, [260, 10], [1, 1], 1),
    ("bf16", 8, 8, 64, 128, [2100, 3, 777], [1, 30, 200], 16),
]


@pytest.mark.parametrize("i", range(len(MASS)))
@pytest.mark.parametrize("keep,in_place", [(1.0, False), (0.9375, True), (0.0, False)])
def test_mass(i, keep, in_place):
    dt, hq, hk, dh, page, cached, new, window = MASS[i]
    rng = np.random.default_rng(i * 3 + in_place)
    s = setup_mass(rng, dt, hq, hk, dh, page, cached, new, pad=16 * (i % 2))
    mass_in = torch.from_numpy(rng.random((len(cached), s["ld"])).astype(np.float32) * 4).to(cuda())
    gone = [int(v) for v in rng.integers(0, 900, len(cached))] if i % 3 else None
    out, birth = run_mass(s, dt, hq, hk, dh, page, window, keep, mass_in, gone, in_place=in_place)
    check_mass(s, out, birth, dt, hq, hk, dh, page, window, keep, mass_in, gone, untouched=None if in_place else -3.0)
    again, _ = run_mass(s, dt, hq, hk, dh, page, window, keep, mass_in, gone, in_place=in_place, ws_fill=0)
    assert torch.equal(out, again)
    if keep == 0.0:                              # each softmax's weights add up to 1
        for b, n in enumerate(new):
            total = float(out[b, :s["kv_len"][b]].double().sum())
            assert abs(total - min(n, window) * hq) <= 1e-4 * max(1, min(n, window) * hq)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,hq,hk,dh", [("f32", 4, 2, 64), ("bf16", 8, 2, 128), ("f16", 2, 2, 64)])
@pytest.mark.parametrize("window", [1, 3, 40])
def test_mass_of_accepted_rows(dt, hq, hk, dh, window):
    rng = np.random.default_rng(window)
    new, accepted = [24, 7, 1, 40, 5], [[0, 3, 4, 20], [6], [0], sorted(rng.permutation(40)[:21].tolist()), []]
    s = setup_mass(rng, dt, hq, hk, dh, 16, [100, 0, 7, 300, 20], new, accepted)
    mass_in = torch.from_numpy(rng.random((5, s["ld"])).astype(np.float32)).to(cuda())
    out, birth = run_mass(s, dt, hq, hk, dh, 16, window, 1.0, mass_in, [3, 0, 5, 0, 0], accepted, draft=30)
    check_mass(s, out, birth, dt, hq, hk, dh, 16, window, 1.0, mass_in, [3, 0, 5, 0, 0], accepted)
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,hq,hk,dh", [("f32", 4, 2, 64), ("bf16", 8, 2, 128), ("f16", 4, 4, 64)])
@pytest.mark.parametrize("new,window", [([3, 4], 4), ([30, 50], 50)])
def test_mass_does_not_see_hidden_keys(dt, hq, hk, dh, new, window):
    """Infinite and NaN keys behind a request's end, in other rows of its pages, and among the new rows that
    only later rows see."""
    rng = np.random.default_rng(11)
    cached, page = [61, 130], 16
    s = setup_mass(rng, dt, hq, hk, dh, page, cached, new)
    used = np.concatenate([[s["table"][b][t // page] * page + t % page for t in range(kv)] for b, kv in enumerate(s["kv_len"])])
    rest = np.setdiff1d(np.arange(s["n_pages"] * page), used)
    s["kv"][torch.from_numpy(rest).to(cuda())] = math.nan
    s["kv"][torch.from_numpy(rest[::2]).to(cuda())] = math.inf
    s["kv"][:, hk * dh:] = math.nan               # values are not looked at
    mass_in = torch.ones(2, s["ld"], device=cuda())
    out, birth = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, None)
    check_mass(s, out, birth, dt, hq, hk, dh, page, window, 1.0, mass_in, None)
    # the last key of request 0 is NaN: its last row's weights are NaN, no other request's
    t = s["kv_len"][0] - 1
    s["kv"][s["table"][0][t // page] * page + t % page, :dh] = math.nan
    out, _ = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, None)
    assert out[0, :t + 1].isnan().all() and not out[1, :s["kv_len"][1]].isnan().any()
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("dt,window,new", [("f32", 2, 2), ("bf16", 2, 2), ("bf16", 40, 40)])
def test_mass_of_large_scores(dt, window, new):
    """Scores of some thousands: a softmax that is one key's."""
    rng = np.random.default_rng(5)
    s = setup_mass(rng, dt, 4, 2, 64, 16, [300, 77], [new, new], size=2000.0)
    mass_in = torch.zeros(2, s["ld"], device=cuda())
    out, _ = run_mass(s, dt, 4, 2, 64, 16, window, 0.0, mass_in, None)
    for b in range(2):
        total = float(out[b, :s["kv_len"][b]].double().sum())
        assert abs(total - new * 4) < 1e-3 and bool((out[b, :s["kv_len"][b]] >= 0).all())
    minus = s["q"].clone()
    s["q"], s["kv"] = torch.full_like(minus, -1e4), s["kv"].abs() + 0.5   # every score far below zero
    out, _ = run_mass(s, dt, 4, 2, 64, 16, window, 0.0, mass_in, None)
    for b in range(2):
        assert abs(float(out[b, :s["kv_len"][b]].double().sum()) - new * 4) < 1e-3


@pytest.mark.parametrize("dt,window", [("f32", 2), ("bf16", 2), ("bf16", 30)])
def test_mass_leaves_inconsistent_requests_out(dt, window):
    rng = np.random.default_rng(8)
    hq, hk, dh, page = 4, 2, 64, 16
    new = [2, 1, 3]
    for kind in ("kv_short", "kv_long", "negative", "offsets", "page"):
        s = setup_mass(rng, dt, hq, hk, dh, page, [40, 50, 60], new)
        good = [0, 2]
        mass_in = torch.rand(3, s["ld"], device=cuda())
        want, _ = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, None)
        cap = sum(s["kv_len"])
        if kind == "kv_short":
            s["kv_len"][1] = 0
        elif kind == "kv_long":
            s["kv_len"][1] = s["ld"] + 1
        elif kind == "negative":
            s["kv_len"][1] = -5
        elif kind == "offsets":
            s["cu"][1], good = 99, []
        else:
            s["table"][1][1], good = s["n_pages"] + 5, [0, 2]
        got, _ = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, None, T_kv_cap=cap)
        for b in good:
            assert torch.equal(got[b], want[b]), (kind, b)
        if kind in ("kv_short", "kv_long", "negative"):
            assert (got[1] == -3).all()
        assert S.seer_check_device() == 2, kind


@pytest.mark.parametrize("dt,window", [("f32", 1), ("bf16", 1), ("bf16", 20)])
def test_mass_past_the_key_capacity(dt, window):
    rng = np.random.default_rng(8)
    s = setup_mass(rng, dt, 4, 2, 64, 16, [300, 400, 500, 30], [1, 1, 1, 1])
    mass_in = torch.rand(4, s["ld"], device=cuda())
    want, _ = run_mass(s, dt, 4, 2, 64, 16, window, 1.0, mass_in, None)
    assert S.seer_check_device() == 0
    got, _ = run_mass(s, dt, 4, 2, 64, 16, window, 1.0, mass_in, None, T_kv_cap=702)
    assert torch.equal(got[:2], want[:2]) and (got[2:] == -3).all()
    assert S.seer_check_device() == 5


@pytest.mark.parametrize("dt,hq,window", [("f32", 4, 3), ("bf16", 4, 3), ("bf16", 16, 20)])
def test_mass_records_accepted_entries_outside_the_draft(dt, hq, window):
    rng = np.random.default_rng(9)
    accepted = [[0, 2], [1, 9]]
    s = setup_mass(rng, dt, hq, 2, 64, 16, [40, 50], [3, 4], accepted)
    mass_in = torch.zeros(2, s["ld"], device=cuda())
    out, _ = run_mass(s, dt, hq, 2, 64, 16, window, 0.0, mass_in, None, accepted)
    assert S.seer_check_device() == 2
    assert abs(float(out[0, :42].sum()) - 2 * hq) < 1e-3 and abs(float(out[1, :52].sum()) - hq) < 1e-3


@pytest.mark.parametrize("dt,window,B", [("f32", 1, 700), ("bf16", 1, 2000), ("bf16", 30, 300)])
def test_mass_of_many_short_requests(dt, window, B):
    rng = np.random.default_rng(B)
    cached, new = [int(v) for v in rng.integers(0, 40, B)], [int(v) for v in rng.integers(0, 3, B)]
    s = setup_mass(rng, dt, 2, 1, 64, 8, cached, new)
    mass_in = torch.from_numpy(rng.random((B, s["ld"])).astype(np.float32)).to(cuda())
    out, birth = run_mass(s, dt, 2, 1, 64, 8, window, 1.0, mass_in, None)
    check_mass(s, out, birth, dt, 2, 1, 64, 8, window, 1.0, mass_in, None)


@pytest.mark.parametrize("dt,hq,window,n", [("bf16", 8, 1, 1), ("f32", 2, 2, 2), ("f16", 8, 16, 16)])
def test_mass_over_a_long_cache(dt, hq, window, n):
    rng = np.random.default_rng(n)
    s = setup_mass(rng, dt, hq, 2, 64, 64, [40000, 5, 9000], [n, n, n])
    mass_in = torch.from_numpy(rng.random((3, s["ld"])).astype(np.float32)).to(cuda())
    out, birth = run_mass(s, dt, hq, 2, 64, 64, window, 1.0, mass_in, None)
    check_mass(s, out, birth, dt, hq, 2, 64, 64, window, 1.0, mass_in, None)


# ------------------------------------------------------------------ the choice of rows
def births(rng, n, gone, tail):
    tail = min(tail, n)
    early = rng.permutation(n - tail + gone)[:n - tail]
    return np.concatenate([early, np.arange(n - tail + gone, n + gone)]).astype(np.int64)


def run_select(mass, birth, kv_len, gone, budget, sinks, recent, ld_move, in_place=False):
    B = len(kv_len)
    t = dict(len=i32([-7] * B), gone=i32([-7] * B), n=i32([-7] * B),
             src=torch.full((B, ld_move), -7, dtype=torch.int32, device=cuda()), to=torch.full((B, ld_move), -7, dtype=torch.int32, device=cuda()))
    kv, g = i32(kv_len), None if gone is None else i32(gone)
    if in_place:
        t["len"], t["gone"] = kv, g
    S.seer_evict_select(mass, birth, mass.shape[1], kv, g, i32(budget), B, sinks, recent, t["len"], t["gone"], t["n"], t["src"], t["to"], ld_move)
    return {k: v.cpu().numpy() for k, v in t.items()}


@pytest.mark.parametrize("B,top,sinks,recent,kind", [
    (1, 1, 0, 0, "plain"), (5, 40, 4, 8, "plain"), (40, 700, 4, 64, "plain"), (3, 5000, 2, 512, "plain"), (2, 70000, 4, 64, "plain"),
    (1, 150000, 0, 10000, "plain"), (9, 300, 0, 0, "ties"), (2, 20000, 4, 32, "ties"), (4, 900, 1, 7, "odd"), (300, 90, 4, 16, "plain"),
    (3, 3000, 50, 100000, "plain"), (2, 9000, 5000, 0, "plain")])
def test_select(B, top, sinks, recent, kind):
    rng = np.random.default_rng(B * 31 + top)
    kv_len = [int(v) for v in rng.integers(0, top + 1, B)]
    kv_len[0] = top
    gone = [int(v) for v in rng.integers(0, 2, B) * rng.integers(1, 5000, B)]
    budget = [int(v) for v in rng.integers(0, max(2, top + top // 8), B)]
    budget[0] = max(1, top // 3)
    if B > 4:
        budget[1], budget[2], budget[3] = 0, kv_len[2], max(0, kv_len[3] - 1)
    ld = top + 3
    mass = np.exp(rng.standard_normal((B, ld)) * 3).astype(np.float32)
    if kind == "ties":
        mass = rng.integers(0, 4, (B, ld)).astype(np.float32)
        mass[mass == 0] *= rng.choice([-1.0, 1.0], int((mass == 0).sum()))    # zeros of both signs
    if kind == "odd":
        mass[rng.random((B, ld)) < 0.2] = math.nan
        mass[rng.random((B, ld)) < 0.1] = math.inf
        mass[rng.random((B, ld)) < 0.1] = -math.inf
        mass[rng.random((B, ld)) < 0.1] *= -1
    birth = np.full((B, ld), -1)
    for b in range(B):
        birth[b, :kv_len[b]] = births(rng, kv_len[b], gone[b], max(recent, 10)) if gone[b] else np.arange(kv_len[b])
    ld_move = max([min(min(k, n), n - min(k, n)) for k, n in zip(budget, kv_len)] + [1])
    got = run_select(torch.from_numpy(mass).to(cuda()), i32(birth), kv_len, gone, budget, sinks, recent, ld_move, in_place=B % 2 == 0)
    for b in range(B):
        k, g, src, to = R.select(mass[b], birth[b], kv_len[b], gone[b], budget[b], sinks, recent)
        assert (got["len"][b], got["gone"][b], got["n"][b]) == (k, g, len(src)), b
        assert got["src"][b, :len(src)].tolist() == src and got["to"][b, :len(to)].tolist() == to, b
        assert (got["src"][b, len(src):] == -7).all() and (got["to"][b, len(to):] == -7).all()
    assert S.seer_check_device() == 0


@pytest.mark.parametrize("ld", [100, 50000])
def test_select_leaves_inconsistent_requests_as_they_are(ld):
    kv_len, budget = [40, -3, ld + 1, 40, 40], [30, 10, 10, -1, 20]
    mass, birth = torch.rand(5, ld, device=cuda()), torch.arange(ld, dtype=torch.int32, device=cuda()).repeat(5, 1)
    got = run_select(mass, birth, kv_len, None, budget, 0, 0, 10)
    assert got["len"].tolist() == [30, -3, ld + 1, 40, 40] and got["n"].tolist()[1:] == [0, 0, 0, 0]
    assert got["gone"].tolist() == [10, 0, 0, 0, 0]
    assert S.seer_check_device() in (2, 5)
    got = run_select(mass[:1].contiguous(), birth[:1].contiguous(), [40], None, [20], 0, 0, 10)   # up to 20 moves, room for 10
    assert got["len"].tolist() == [40] and got["n"].tolist() == [0] and S.seer_check_device() == 5


# ------------------------------------------------------------------ the moves
@pytest.mark.parametrize("dt,hk,dh", [("bf16", 8, 128), ("f32", 1, 8), ("f16", 3, 80), ("f32", 5, 128)])
@pytest.mark.parametrize("B,top,page", [(1, 1, 8), (4, 528, 16), (7, 3000, 64), (200, 60, 8)])
def test_evict(dt, hk, dh, B, top, page):
    rng = np.random.default_rng(top + dh)
    kv_len = [int(v) for v in rng.integers(0, top + 1, B)]
    kv_len[0] = top
    s = setup_mass(rng, dt, hk, hk, dh, page, kv_len, [0] * B)
    moves = []
    for n in kv_len:
        k = int(rng.integers(0, n + 1))
        m = int(rng.integers(0, min(k, n - k) + 1))
        moves.append((sorted(rng.permutation(np.arange(k, n))[:m].tolist()), sorted(rng.permutation(k)[:m].tolist())))
    ld_move = max([len(m[0]) for m in moves]) + 2
    src, to = (i32([m[e] + [-1] * (ld_move - len(m[e])) for m in moves]) for e in (0, 1))
    mass = torch.from_numpy(rng.random((B, s["ld"])).astype(np.float32)).to(cuda())
    birth = torch.arange(B * s["ld"], dtype=torch.int32, device=cuda()).view(B, -1)
    kv, m0, b0 = s["kv"].clone(), mass.clone(), birth.clone()
    table = i32(s["table"])
    pages = S.make_pages(s["kv"], table, s["n_pages"], page, s["max_pages"], hk, dh)
    S.seer_kv_evict(dt, i32(kv_len), i32([len(m[0]) for m in moves]), src, to, ld_move, B, pages, mass, birth, s["ld"])
    for b, (f, t) in enumerate(moves):
        rows = [torch.tensor([int(s["table"][b][x // page]) * page + x % page for x in part], dtype=torch.long, device=cuda()) for part in (f, t)]
        kv[rows[1]] = kv[rows[0]]
        m0[b, t], b0[b, t] = m0[b, f], b0[b, f]
    assert torch.equal(s["kv"], kv) and torch.equal(mass, m0) and torch.equal(birth, b0)
    assert S.seer_check_device() == 0


def test_evict_leaves_bad_moves_out():
    rng = np.random.default_rng(1)
    s = setup_mass(rng, "f32", 1, 1, 8, 8, [30, 30, 30], [0, 0, 0])
    s["table"][2][3] = 10 ** 6
    kv, mass = s["kv"].clone(), torch.rand(3, s["ld"], device=cuda())
    m0 = mass.clone()
    src, to = i32([[29, 30, -1, 25], [28, 27, 26, 25], [29, 20, 0, 0]]), i32([[2, 3, 4, 500], [0, 1, 2, 3], [0, 1, 0, 0]])
    table = i32(s["table"])
    pages = S.make_pages(s["kv"], table, s["n_pages"], 8, s["max_pages"], 1, 8)
    S.seer_kv_evict("f32", i32([30, 30, 30]), i32([4, 5, 2]), src, to, 4, 3, pages, mass, None, s["ld"])
    assert S.seer_check_device() == 2

    def row(b, t):
        return int(s["table"][b][t // 8]) * 8 + t % 8
    kv[row(0, 2)], m0[0, 2] = kv[row(0, 29)], m0[0, 29]
    kv[row(2, 1)], m0[2, 1] = kv[row(2, 20)], m0[2, 20]
    assert torch.equal(s["kv"], kv) and torch.equal(mass, m0)


# ------------------------------------------------------------------ together
class Server:
    """A layer's cache kept within budgets, a step at a time, and its statement in plain Python."""

    def __init__(self, dt, hq, hk, dh, page, B, pages, max_pages, budget, sinks, recent, rot, rate, inter, seed):
        self.rng = np.random.default_rng(seed)
        self.__dict__.update(dt=dt, hq=hq, hk=hk, dh=dh, page=page, B=B, n_pages=pages, max_pages=max_pages, budget=budget, sinks=sinks,
                             recent=recent, rot=rot, rate=rate, inter=inter)
        self.kv = torch.zeros(pages * page, 2 * hk * dh, dtype=TDT[dt], device=cuda())
        self.table = torch.full((B, max_pages), -1, dtype=torch.int32, device=cuda())
        self.pages = S.make_pages(self.kv, self.table, pages, page, max_pages, hk, dh)
        self.ld = max_pages * page
        self.mass = torch.zeros(B, self.ld, device=cuda())
        self.birth = torch.full((B, self.ld), -1, dtype=torch.int32, device=cuda())
        self.cached, self.gone = [0] * B, [0] * B
        self.free = list(range(pages))
        # the statement: per request its rows in cache order (key, value, mass, birth)
        self.rows = [[] for _ in range(B)]

    def step(self, new, window):
        hq, hk, dh, B = self.hq, self.hk, self.dh, self.B
        T = sum(new)
        x = rnd(self.rng, (T, (hq + 2 * hk) * dh), self.dt)
        cu, kv_len, slot, pos, head = i32([0] * (B + 1)), i32([0] * B), i32([0] * T), i32([0] * T), i32([0])
        S.seer_page_tables(i32(self.cached), i32(new), B, self.page, self.n_pages, i32(self.free), len(self.free), i32([0]), self.table,
                           self.max_pages, T, None, cu, kv_len, slot, pos, None, head)
        self.free = self.free[int(head[0]):]
        qk = torch.zeros(T, (hq + hk) * dh, dtype=TDT[self.dt], device=cuda())
        S.seer_kv_append_rotary(x, x.stride(0), self.dt, hq, T, None, slot, pos, cu, i32(self.gone), B, self.rot, qk, qk.stride(0), self.pages)
        o = torch.zeros(T, hq * dh, dtype=TDT[self.dt], device=cuda())
        draft = max(new)
        need = S.seer_attention_tree_workspace_size(self.dt, B, hq, hk, dh, draft)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=cuda())
        S.seer_attention_tree(qk, qk.stride(0), o, o.stride(0), self.dt, cu, kv_len, None, B, T, hq, draft, self.pages, ws, need)
        cap = sum(self.cached) + T
        need = S.seer_attention_mass_workspace_size(self.dt, B, cap, hq, hk, dh, window)
        ws = torch.empty(need, dtype=torch.uint8, device=cuda())
        S.seer_attention_mass(qk, qk.stride(0), self.dt, cu, kv_len, None, None, 0, window, B, T, cap, hq, self.pages, 1.0, i32(self.gone),
                              self.mass, self.mass, self.birth, self.ld, ws, need)
        # the statement's new rows: turned by the positions since the request's start
        xs = host(x).reshape(T, hq + 2 * hk, dh)
        at = np.concatenate([c + g + np.arange(n) for c, g, n in zip(self.cached, self.gone, new)])
        turned = R.turn(xs[:, :hq + hk], at, self.rate, self.inter)
        bound = R.turn_bound(xs[:, :hq + hk], turned, at, 2 * len(self.rate), self.inter, self.dt)
        close(qk.reshape(T, hq + hk, dh), turned, bound, "rotated")
        # attention and mass from the rows as they are stored, so that only their own roundings count
        got = host(qk).reshape(T, hq + hk, dh)
        r = 0
        for b, n in enumerate(new):
            self.rows[b] += [[got[r + i, hq:], xs[r + i, hq + hk:], 0.0, 0.0, int(at[r + i])] for i in range(n)]
            if n:
                k, v = (np.stack([row[e] for row in self.rows[b]]) for e in (0, 1))
                c = len(self.rows[b]) - n
                seen = np.concatenate([np.ones((n, c), bool), np.tril(np.ones((n, n), bool))], 1)
                for h in range(hq):
                    ref, bound = PR.attend(got[r:r + n, h], k[:, h * hk // hq], v[:, h * hk // hq], seen, self.dt)
                    close(o[r:r + n, h * dh:(h + 1) * dh], ref, bound, "attention")
                look = list(range(max(0, n - window), n))
                (w, err), = R.mass(got[r:r + n, :hq], k, [[0]], 1 << 30, [(look, look, n, len(k))], 1.0, [[row[2] for row in self.rows[b][:c]]], dh)
                for row, a, e in zip(self.rows[b], w, err):
                    row[2], row[3] = a, row[3] + e + abs(a) * 2.0 ** -23
                close(self.mass[b, :len(w)], w, np.array([row[3] for row in self.rows[b]]), "mass")
                assert self.birth[b, :len(w)].tolist() == [row[4] for row in self.rows[b]]
            r += n
        self.cached = kv_len.tolist()

    def evict(self):
        B = self.B
        ld_move = max(min(k, n - min(k, n)) for k, n in zip(self.budget, self.cached)) + 1
        kv_len, gone = i32(self.cached), i32(self.gone)
        out = [i32([0] * B) for _ in range(3)] + [torch.zeros(B, ld_move, dtype=torch.int32, device=cuda()) for _ in range(2)]
        S.seer_evict_select(self.mass, self.birth, self.ld, kv_len, gone, i32(self.budget), B, self.sinks, self.recent, *out, ld_move)
        S.seer_kv_evict(self.dt, kv_len, out[2], out[3], out[4], ld_move, B, self.pages, self.mass, self.birth, self.ld)
        mass = host(self.mass)
        for b in range(B):
            n = self.cached[b]
            before = self.mass_before(b, mass, out, n)
            k, g, src, to = R.select(before, [row[4] for row in self.rows[b]], n, self.gone[b], self.budget[b], self.sinks, self.recent)
            assert (int(out[0][b]), int(out[1][b]), int(out[2][b])) == (k, g, len(src))
            assert out[3][b, :len(src)].tolist() == src and out[4][b, :len(to)].tolist() == to
            for f, t in zip(src, to):
                self.rows[b][t] = self.rows[b][f]
            del self.rows[b][k:]
            held = self.table[b, -(-k // self.page):-(-n // self.page)].tolist()
            self.free += held
        self.cached, self.gone = out[0].tolist(), out[1].tolist()

    @staticmethod
    def mass_before(b, mass, out, n):
        """A request's masses before its moves: the rows moved to lost theirs, which is below what stayed."""
        before = mass[b, :n].copy()
        m = int(out[2][b])
        before[out[4][b, :m].tolist()] = -1.0
        return before


@pytest.mark.parametrize("dt,inter,scaling,dh", [("bf16", True, "turns", 64), ("f32", False, "pairs", 64), ("f16", False, "linear", 128)])
def test_a_server_keeps_to_its_budgets(dt, inter, scaling, dh):
    rot, rate = rotary(10000.0, dh // 2, inter, scaling)
    s = Server(dt, 4, 2, dh, 8, 3, 60, 16, [40, 25, 33], 2, 6, rot, rate, inter, 17)
    s.step([50, 30, 9], 8)
    s.evict()
    for i in range(6):
        s.step([1, 3, 5] if i % 2 else [1, 1, 0], 8)
        if i != 2:                                # a step without eviction: the cache runs over its budget and comes back
            s.evict()
        assert all(len(set(row[4] for row in rows)) == len(rows) for rows in s.rows)
    assert s.cached[0] == 40 and s.gone[0] == 50 + 6 - 40
    for b in range(3):                            # sinks and the last rows are there
        born = {row[4] for row in s.rows[b]}
        last = s.cached[b] + s.gone[b]
        assert {0, 1} <= born and set(range(last - 6, last)) <= born
    assert S.seer_check_device() == 0


# ------------------------------------------------------------------ streams and graphs
def test_two_captured_steps_replay_with_their_own_lengths():
    """A step captured once goes on with the lengths on the device; two graphs have a workspace each."""
    rng = np.random.default_rng(2)
    dt, hq, hk, dh, page, B, window = "bf16", 8, 2, 64, 16, 3, 1
    graphs = []
    for g in range(2):
        s = setup_mass(rng, dt, hq, hk, dh, page, [90, 40, 300], [1, 1, 1])
        table = i32(s["table"])
        pages = S.make_pages(s["kv"], table, s["n_pages"], page, s["max_pages"], hk, dh)
        need = S.seer_attention_mass_workspace_size(dt, B, sum(s["kv_len"]), hq, hk, dh, window)
        t = dict(s=s, table=table, pages=pages, ws=torch.empty(need, dtype=torch.uint8, device=cuda()), need=need, cu=i32(s["cu"]), kv=i32(s["kv_len"]),
                 gone=i32([5, 0, 7]), mass=torch.rand(B, s["ld"], device=cuda()), birth=torch.zeros(B, s["ld"], dtype=torch.int32, device=cuda()),
                 budget=i32([50, 30, 100]), out=[i32([0] * B) for _ in range(3)],
                 moves=[torch.zeros(B, 200, dtype=torch.int32, device=cuda()) for _ in range(2)])
        t["birth"][:] = torch.arange(s["ld"], dtype=torch.int32, device=cuda())

        def step(t=t, s=s):
            S.seer_attention_mass(s["q"], s["q"].stride(0), dt, t["cu"], t["kv"], None, None, 0, window, B, 3, sum(s["kv_len"]), hq, t["pages"],
                                  1.0, t["gone"], t["mass"], t["mass"], t["birth"], s["ld"], t["ws"], t["need"])
            S.seer_evict_select(t["mass"], t["birth"], s["ld"], t["kv"], t["gone"], t["budget"], B, 2, 4, t["out"][0], t["out"][1], t["out"][2],
                                *t["moves"], 200)
            S.seer_kv_evict(dt, t["kv"], t["out"][2], *t["moves"], 200, B, t["pages"], t["mass"], t["birth"], s["ld"])
        t["start"] = [x.clone() for x in (s["kv"], t["mass"], t["birth"])]
        step()
        torch.cuda.synchronize()
        t["want"] = [x.clone() for x in (s["kv"], t["mass"], t["birth"], *t["out"])]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append((graph, t))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _, t in graphs:
        for x, y in zip((t["s"]["kv"], t["mass"], t["birth"]), t["start"]):
            x.copy_(y)
    torch.cuda.synchronize()
    for st, (graph, _) in zip(streams, graphs):
        with torch.cuda.stream(st):
            graph.replay()
    torch.cuda.synchronize()
    for _, t in graphs:
        for x, y in zip((t["s"]["kv"], t["mass"], t["birth"], *t["out"]), t["want"]):
            assert torch.equal(x, y)
    # the same graph with other lengths
    graph, t = graphs[0]
    t["kv"].copy_(i32([20, 41, 10]))
    t["mass"].copy_(t["start"][1])
    graph.replay()
    torch.cuda.synchronize()
    assert t["out"][0].tolist() == [20, 30, 10] and S.seer_check_device() == 0


def test_calls_on_another_stream():
    rng = np.random.default_rng(4)
    s = setup_mass(rng, "bf16", 4, 2, 64, 16, [90, 40], [1, 1])
    mass_in = torch.rand(2, s["ld"], device=cuda())
    want, _ = run_mass(s, "bf16", 4, 2, 64, 16, 1, 1.0, mass_in, None)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        got, _ = run_mass(s, "bf16", 4, 2, 64, 16, 1, 1.0, mass_in, None)
    st.synchronize()
    assert torch.equal(got, want)
