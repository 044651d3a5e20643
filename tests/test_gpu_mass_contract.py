"""What the attention mass promises where keys are odd, capacities end and calls follow one another."""
import math

import numpy as np
import pytest
import torch

from tests.helpers import cuda, i32
from tests.test_gpu_budget import close, host, rnd, run_mass, setup_mass

pytestmark = pytest.mark.gpu

S = pytest.importorskip("paper_2607_14557_gb300.seer")
# dt, hq, hk, window: fp32, few columns, many columns (tensor cores)
PATHS = [("f32", 8, 2, 12), ("bf16", 8, 2, 4), ("f16", 16, 2, 40), ("bf16", 16, 2, 12)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    S.seer_check_device()
    yield
    torch.cuda.synchronize()


def pool_row(s, b, t, page):
    return int(s["table"][b][t // page]) * page + t % page


def expected(s, b, looking, hq, hk, dh, page, odd=()):
    """New weight of request b's rows and how far off it may be.  looking: (row of q, last row that it sees)
    pairs; odd: rows that score minus infinity.

    An exponent is off by the products' chain (dh 2^-24 sum |q k|) and by the roundings of scale,
    score, maximum and difference (2^-21 of the largest score: 2 of 2^-24 of it, 3 of the difference,
    which is at most twice it), in numerator and sum alike; exponentials by 2^-21, the sum of n terms and
    its reciprocal by (n + 4) 2^-24, the sum over columns by one rounding a term.  What fp32 cannot hold
    is below 1e-30 (added by close)."""
    at = np.array([pool_row(s, b, t, page) for t in range(s["kv_len"][b])], int)
    q = host(s["q"])[:, :hq * dh].reshape(-1, hq, dh) / math.sqrt(dh)
    keys = host(s["kv"])[:, :hk * dh].reshape(-1, hk, dh)[at]
    keys[list(odd)] = 0
    w, err = np.zeros(len(at)), np.zeros(len(at))
    for row, last in looking:
        seen = last + 1
        for h in range(hq):
            k = keys[:seen, h // (hq // hk)]
            x, size = k @ q[row, h], (np.abs(k) @ np.abs(q[row, h])).max()
            x[[t for t in odd if t < seen]] = -np.inf
            e = np.exp(x - x.max())
            p = e / e.sum()
            w[:seen] += p
            err[:seen] += p * (np.expm1(2 * (dh * 2.0 ** -24 + 2.0 ** -21) * size) + 2.0 ** -20 + (seen + 4) * 2.0 ** -24)
    return w, err + w * (hq * max(len(looking), 1) + 1) * 2.0 ** -24


def all_looking(s, b, window):
    n, kv, q0 = int(s["cu"][b + 1] - s["cu"][b]), s["kv_len"][b], int(s["cu"][b])
    return [(q0 + i, kv - n + i) for i in range(max(0, n - window), n)]


def odd_key(s, b, t, page, hk, dh, value):
    s["kv"][pool_row(s, b, t, page), :hk * dh] = value


# ------------------------------------------------------------------ rows that do not look
@pytest.mark.parametrize("dt,hq,hk,window", PATHS)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_rows_outside_the_draft_do_not_look_at_odd_keys(dt, hq, hk, window, value):
    """Their queries are nothing, and nothing times an infinite or NaN key is NaN."""
    rng = np.random.default_rng(window)
    dh, page = 64, 16
    accepted = [[0, 2, 70], [66, 67, 68, 69], [1, 65, 3, 4], [70]]
    s = setup_mass(rng, dt, hq, hk, dh, page, [300, 290, 500, 0], [6, 5, 6, 2], accepted)
    s["q"][:, ::dh] = -s["q"][:, ::dh].abs() - 0.25
    odd_key(s, 0, 302, page, hk, dh, value)      # the row that would see it is outside
    odd_key(s, 1, 7, page, hk, dh, value)        # nobody looks, neither here nor in request 3
    odd_key(s, 1, 293, page, hk, dh, value)
    odd_key(s, 3, 0, page, hk, dh, value)
    for t in (3, 200):                           # minus infinity for all that look
        s["kv"][pool_row(s, 2, t, page), :hk * dh:dh] = math.inf
    mass_in = torch.from_numpy(rng.random((4, s["ld"])).astype(np.float32)).to(cuda())
    out, _ = run_mass(s, dt, hq, hk, dh, page, window, 0.0, mass_in, None, accepted, draft=6)
    assert S.seer_check_device() == 2
    q0 = [int(c) for c in s["cu"]]
    for b, looking, odd in ((0, [(q0[0], 300), (q0[0] + 2, 301)], [302]), (1, [], [7, 293]),
                            (2, [(q0[2] + 1, 500), (q0[2] + 3, 502), (q0[2] + 4, 503)], [3, 200]), (3, [], [0])):
        w, err = expected(s, b, looking, hq, hk, dh, page, odd)
        close(out[b, :s["kv_len"][b]], w, err, f"request {b}")
        assert (out[b, odd] == 0).all()


# ------------------------------------------------------------------ the key capacity
@pytest.mark.parametrize("dt,hq,hk,window", PATHS)
def test_the_key_capacity_is_counted_in_keys(dt, hq, hk, window):
    rng = np.random.default_rng(3)
    s = setup_mass(rng, dt, hq, hk, 64, 16, [63, 63, 0, 62, 0, 9], [1, 1, 0, 2, 0, 1])
    mass_in = torch.rand(6, s["ld"], device=cuda())
    want, _ = run_mass(s, dt, hq, hk, 64, 16, window, 1.0, mass_in, None)
    assert S.seer_check_device() == 0 and sum(s["kv_len"]) == 202
    for cap, served in ((202, 6), (201, 5), (192, 5), (191, 3), (128, 3), (127, 1), (64, 1), (63, 0), (0, 0)):
        got, birth = run_mass(s, dt, hq, hk, 64, 16, window, 1.0, mass_in, None, T_kv_cap=cap)
        assert torch.equal(got[:served], want[:served]), cap
        assert (got[served:] == -3).all() and (birth[served:] == -9).all(), cap
        assert S.seer_check_device() == (0 if cap == 202 else 5), cap


@pytest.mark.parametrize("dt,hq,hk,window", PATHS)
def test_requests_that_do_not_fit_their_matrix_take_no_capacity(dt, hq, hk, window):
    rng = np.random.default_rng(4)
    s = setup_mass(rng, dt, hq, hk, 64, 16, [100, 40, 30], [1, 1, 1])
    mass_in = torch.rand(3, s["ld"], device=cuda())
    want, _ = run_mass(s, dt, hq, hk, 64, 16, window, 1.0, mass_in, None)
    cap = s["kv_len"][0] + s["kv_len"][2]
    s["kv_len"][1] = 2 ** 31 - 1
    got, _ = run_mass(s, dt, hq, hk, 64, 16, window, 1.0, mass_in, None, T_kv_cap=cap)
    assert torch.equal(got[[0, 2]], want[[0, 2]]) and (got[1] == -3).all() and S.seer_check_device() == 2


@pytest.mark.parametrize("dt,hq,hk,window,B", [("f32", 2, 1, 3, 700), ("bf16", 2, 1, 3, 2000), ("f16", 2, 1, 30, 1500)])
def test_the_key_capacity_ends_inside_a_large_batch(dt, hq, hk, window, B):
    rng = np.random.default_rng(B)
    cached, new = [int(v) for v in rng.integers(0, 40, B)], [int(v) for v in rng.integers(0, 3, B)]
    s = setup_mass(rng, dt, hq, hk, 64, 8, cached, new)
    mass_in = torch.rand(B, s["ld"], device=cuda())
    want, _ = run_mass(s, dt, hq, hk, 64, 8, window, 1.0, mass_in, None)
    ends = np.cumsum(s["kv_len"])
    for served in (B // 3, B - 2):
        while s["kv_len"][served] == 0:          # (the first that is left out has keys)
            served += 1
        for cap in (int(ends[served - 1]), int(ends[served]) - 1):
            got, _ = run_mass(s, dt, hq, hk, 64, 8, window, 1.0, mass_in, None, T_kv_cap=cap)
            assert torch.equal(got[:served], want[:served]) and (got[served:] == -3).all()
            assert S.seer_check_device() == 5


# ------------------------------------------------------------------ infinite scores of rows that look
@pytest.mark.parametrize("dt,hq,hk,window", PATHS)
def test_infinite_scores(dt, hq, hk, window):
    """Minus infinity weighs nothing; plus infinity, or nothing but minus infinity, makes the row's
    weights NaN for what it sees."""
    rng = np.random.default_rng(6)
    dh, page, new = 64, 16, [3, 2, 1, 4, 2]
    s = setup_mass(rng, dt, hq, hk, dh, page, [400, 300, 0, 200, 77], new)
    s["q"][:, ::dh] = -s["q"][:, ::dh].abs() - 0.25
    lowest = [0, 64, 399, 400]
    for t in lowest:
        s["kv"][pool_row(s, 0, t, page), :hk * dh:dh] = math.inf
    s["kv"][pool_row(s, 1, 130, page), :hk * dh:dh] = -math.inf
    s["kv"][pool_row(s, 2, 0, page), :hk * dh:dh] = math.inf
    s["kv"][pool_row(s, 3, 202, page), :hk * dh:dh] = -math.inf     # of the last two rows' alone
    mass_in = torch.from_numpy(rng.random((5, s["ld"])).astype(np.float32)).to(cuda())
    out, _ = run_mass(s, dt, hq, hk, dh, page, window, 0.0, mass_in, None)
    for b, odd in ((0, lowest), (4, [])):
        w, err = expected(s, b, all_looking(s, b, window), hq, hk, dh, page, odd)
        close(out[b, :s["kv_len"][b]], w, err, f"request {b}")
    assert (out[0, lowest] == 0).all()
    for b in (1, 2, 3):
        assert out[b, :s["kv_len"][b]].isnan().all()
    assert S.seer_check_device() == 0


# ------------------------------------------------------------------ scores that leave one key its weight
@pytest.mark.parametrize("dt,hq,hk,window,new", [("f32", 4, 2, 2, 2), ("bf16", 4, 2, 2, 2), ("bf16", 4, 2, 40, 40), ("f16", 4, 4, 3, 3)])
@pytest.mark.parametrize("below", [False, True])
def test_large_scores_key_by_key(dt, hq, hk, window, new, below):
    """Scores of thousands, of either sign, over caches that are cut into many pieces."""
    rng = np.random.default_rng(5)
    dh, page = 64, 16
    s = setup_mass(rng, dt, hq, hk, dh, page, [12000, 300, 77], [new] * 3, size=2000.0)
    if below:
        s["q"], s["kv"] = -(s["q"].abs() / 8 + 300), s["kv"].abs() + 0.5
    mass_in = torch.zeros(3, s["ld"], device=cuda())
    out, _ = run_mass(s, dt, hq, hk, dh, page, window, 0.0, mass_in, None)
    for b in range(3):
        w, err = expected(s, b, all_looking(s, b, window), hq, hk, dh, page)
        assert w.max() > 0.5                                    # few keys hold nearly all of it
        close(out[b, :s["kv_len"][b]], w, err, f"request {b}")
    assert S.seer_check_device() == 0


# ------------------------------------------------------------------ calls behind one another
@pytest.mark.parametrize("dt,hq,hk,window", PATHS)
@pytest.mark.parametrize("overlap", [True, False])
def test_calls_behind_one_another_share_a_workspace(dt, hq, hk, window, overlap):
    """Nothing between the calls but the calls: what one leaves in the workspace is the next one's to
    overwrite as soon as the first has read it, and no sooner."""
    rng = np.random.default_rng(7)
    dh, page = 64, 16
    sets, ws_bytes = [], 0
    for cached, new in (([3000, 33, 0, 700], [window, 1, 2, 1]), ([5, 1200], [1, window]), ([64] * 40, [1] * 40)):
        s = setup_mass(rng, dt, hq, hk, dh, page, cached, new)
        B, cap = len(new), sum(s["kv_len"])
        mass_in = torch.rand(B, s["ld"], device=cuda())
        want, want_birth = run_mass(s, dt, hq, hk, dh, page, window, 0.5, mass_in, [3] * B)
        table, cu, kv_len, gone = i32(s["table"]), i32(s["cu"]), i32(s["kv_len"]), i32([3] * B)
        pages = S.make_pages(s["kv"], table, s["n_pages"], page, s["max_pages"], hk, dh)
        ws_bytes = max(ws_bytes, S.seer_attention_mass_workspace_size(dt, B, cap, hq, hk, dh, window))
        outs = [(torch.full_like(mass_in, -3.0), torch.full(mass_in.shape, -9, dtype=torch.int32, device=cuda())) for _ in range(6)]
        sets.append((s, B, cap, mass_in, table, cu, kv_len, gone, pages, outs, want, want_birth))
    ws = torch.full((ws_bytes,), 255, dtype=torch.uint8, device=cuda())
    was = S.seer_set_launch_overlap(overlap)
    try:
        torch.cuda.synchronize()
        for i in range(6):
            for s, B, cap, mass_in, table, cu, kv_len, gone, pages, outs, _, _ in sets:
                S.seer_attention_mass(s["q"], s["q"].stride(0), dt, cu, kv_len, None, None, 1, window, B, s["q"].shape[0], cap, hq, pages, 0.5,
                                      gone, mass_in, *outs[i], s["ld"], ws, ws_bytes)
        torch.cuda.synchronize()
    finally:
        S.seer_set_launch_overlap(was)
    for *_, outs, want, want_birth in sets:
        for out, birth in outs:
            assert torch.equal(out, want) and torch.equal(birth, want_birth)
    assert S.seer_check_device() == 0


# ------------------------------------------------------------------ a whole prompt's weight
@pytest.mark.parametrize("dt,hq,hk,window", [("f32", 4, 2, 64), ("bf16", 4, 2, 64), ("f16", 4, 4, 16)])
def test_a_whole_prompt_looks_in_calls_of_a_window_each(dt, hq, hk, window):
    """The prompts' rows as lists of accepted ones, a window's worth a call, the cache as long as they reach."""
    rng = np.random.default_rng(8)
    dh, page, new = 64, 16, [3 * window + 5, window, 1, 2 * window - 1]
    s = setup_mass(rng, dt, hq, hk, dh, page, [0] * 4, new)
    B, cap = 4, sum(new)
    table, cu, gone = i32(s["table"]), i32(s["cu"]), i32([0] * B)
    pages = S.make_pages(s["kv"], table, s["n_pages"], page, s["max_pages"], hk, dh)
    n = S.seer_attention_mass_workspace_size(dt, B, cap, hq, hk, dh, window)
    ws = torch.empty(n, dtype=torch.uint8, device=cuda())
    mass, birth = torch.full((B, s["ld"]), -3.0, device=cuda()), torch.full((B, s["ld"]), -9, dtype=torch.int32, device=cuda())
    for at in range(0, max(new), window):
        count = [max(0, min(window, m - at)) for m in new]
        accepted = i32([list(range(at, at + window))] * B)
        S.seer_attention_mass(s["q"], s["q"].stride(0), dt, cu, i32([min(at + window, m) for m in new]), accepted, i32(count), window, window, B,
                              s["q"].shape[0], cap, hq, pages, 1.0, gone, mass, mass, birth, s["ld"], ws, n)
    for b, m in enumerate(new):
        w, err = expected(s, b, [(int(s["cu"][b]) + i, i) for i in range(m)], hq, hk, dh, page)
        close(mass[b, :m], w, err + w * 2.0 ** -24 * 4, f"request {b}")     # (a sum over the calls)
        assert (mass[b, m:] == -3).all() and (birth[b, :m].cpu() == torch.arange(m)).all() and (birth[b, m:] == -9).all()
    assert S.seer_check_device() == 0
