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
