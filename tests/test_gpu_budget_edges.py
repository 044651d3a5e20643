"""The budget operators where sizes, offsets and layouts are unusual."""
import math

import numpy as np
import pytest
import torch

from tests import budget_reference as R
from tests.helpers import cuda, i32
from tests.test_gpu_budget import TDT, check_mass, close, host, rnd, rotary, run_mass, setup_mass

pytestmark = pytest.mark.gpu

S = pytest.importorskip("paper_2607_14557_gb300.seer")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    S.seer_check_device()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dt,hq,hk,dh,page,cached,new,window", [
    ("bf16", 12, 12, 64, 16, [70, 200], [1, 1], 1),            # more heads than warps, not a multiple of them
    ("f16", 40, 20, 128, 8, [33, 100, 0], [2, 1, 3], 3),
    ("bf16", 16, 1, 128, 16, [500, 3], [1, 1], 1),             # 16 columns of one head
    ("f16", 45, 5, 64, 32, [129, 64], [1, 1], 1),
    ("f16", 14, 2, 128, 16, [300, 0, 90], [64, 50, 3], 64),    # several column blocks, groups that do not divide a tile
    ("bf16", 128, 1, 64, 16, [129, 700], [5, 1], 5),
    ("bf16", 9, 9, 128, 64, [1000], [40], 40),
    ("f16", 33, 3, 64, 8, [513, 1], [24, 2], 24),
    ("f32", 24, 12, 24, 8, [77, 300], [5, 30], 30),
    ("f32", 17, 1, 8, 16, [64, 63, 0], [1, 2, 64], 64),
    ("f32", 3, 3, 128, 256, [1000], [1], 1)])
def test_mass_of_unusual_heads(dt, hq, hk, dh, page, cached, new, window):
    rng = np.random.default_rng(hq + window)
    s = setup_mass(rng, dt, hq, hk, dh, page, cached, new)
    mass_in = torch.from_numpy(rng.random((len(cached), s["ld"])).astype(np.float32)).to(cuda())
    out, birth = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, [7] * len(cached))
    check_mass(s, out, birth, dt, hq, hk, dh, page, window, 1.0, mass_in, [7] * len(cached))
    again, _ = run_mass(s, dt, hq, hk, dh, page, window, 1.0, mass_in, [7] * len(cached), ws_fill=0)
    assert torch.equal(out, again) and S.seer_check_device() == 0


@pytest.mark.parametrize("window", [1, 30])
def test_mass_of_a_step_without_rows_fades(window):
    """No request has new rows; q has no address."""
    kv, table = torch.zeros(32, 256, dtype=torch.bfloat16, device=cuda()), i32([[0, 1], [2, 3]])
    mass = torch.rand(2, 20, device=cuda())
    want = mass * 0.5
    want[0, 9:], want[1, 16:] = mass[0, 9:], mass[1, 16:]
    need = S.seer_attention_mass_workspace_size("bf16", 2, 25, 4, 2, 64, window)
    ws = torch.empty(need, dtype=torch.uint8, device=cuda())
    S.seer_attention_mass(None, 256, "bf16", i32([0, 0, 0]), i32([9, 16]), None, None, 0, window, 2, 0, 25, 4, S.make_pages(kv, table, 4, 8, 2, 2, 64), 0.5,
                          None, mass, mass, None, 20, ws, need)
    assert torch.equal(mass, want) and S.seer_check_device() == 0


@pytest.mark.parametrize("dt,hq,window", [("f32", 2, 1), ("bf16", 2, 1), ("bf16", 24, 1)])
def test_mass_of_more_tiles_than_blocks(dt, hq, window):
    """A capacity far above the keys, and more tiles of keys than the second kernel has blocks."""
    rng = np.random.default_rng(3)
    B = 3000
    cached = [int(v) for v in rng.integers(0, 130, B)]
    s = setup_mass(rng, dt, hq, 1, 64, 16, cached, [1] * B)
    mass_in = torch.from_numpy(rng.random((B, s["ld"])).astype(np.float32)).to(cuda())
    want, birth = run_mass(s, dt, hq, 1, 64, 16, window, 1.0, mass_in, None)
    got, _ = run_mass(s, dt, hq, 1, 64, 16, window, 1.0, mass_in, None, T_kv_cap=600000)
    if dt == "f32" or hq * window <= 16:           # (the runs follow from the keys alone)
        assert torch.equal(got, want)
    check_mass(s, got, birth, dt, hq, 1, 64, 16, window, 1.0, mass_in, None)


@pytest.mark.parametrize("dt,hq,window", [("f32", 1, 1), ("f16", 1, 1), ("f16", 17, 1)])
def test_the_most_requests(dt, hq, window):
    """16384 requests of one to three rows: mass, choice and moves."""
    rng = np.random.default_rng(4)
    B, page = S.MAX_REQUESTS, 8
    cached = rng.integers(0, 3, B)
    kv_len = cached + 1
    kv = rnd(rng, (B * page, 2 * 64), dt)
    table = i32(rng.permutation(B)[:, None])
    pages = S.make_pages(kv, table, B, page, 1, 1, 64)
    q = rnd(rng, (B, hq * 64), dt)
    need = S.seer_attention_mass_workspace_size(dt, B, int(kv_len.sum()), hq, 1, 64, window)
    ws = torch.empty(need, dtype=torch.uint8, device=cuda())
    mass, birth = torch.zeros(B, 4, device=cuda()), torch.zeros(B, 4, dtype=torch.int32, device=cuda())
    birth[:] = torch.arange(4, dtype=torch.int32, device=cuda())
    lens = i32(kv_len)
    S.seer_attention_mass(q, hq * 64, dt, i32(np.arange(B + 1)), lens, None, None, 0, window, B, B, int(kv_len.sum()), hq, pages, 1.0, None, mass, mass,
                          birth, 4, ws, need)
    total = mass.double().sum(1)
    assert float((total - hq).abs().max()) < 1e-4 * hq
    out = [i32([0] * B) for _ in range(3)] + [torch.zeros(B, 1, dtype=torch.int32, device=cuda()) for _ in range(2)]
    S.seer_evict_select(mass, birth, 4, lens, None, i32([2] * B), B, 0, 1, *out, 1)
    host_mass, before = host(mass), kv.clone()
    S.seer_kv_evict(dt, lens, out[2], out[3], out[4], 1, B, pages, mass, birth, 4)
    three = np.nonzero(kv_len == 3)[0]                # the last row stays, and the heavier of the others: it moves to row 0 or 1
    weaker = np.where(host_mass[three, 0] >= host_mass[three, 1], 1, 0)
    assert (out[2].cpu().numpy() == (kv_len == 3)).all() and (out[0].cpu().numpy() == np.minimum(kv_len, 2)).all()
    assert (out[3].cpu().numpy()[three, 0] == 2).all() and (out[4].cpu().numpy()[three, 0] == weaker).all()
    at = table[:, 0].long()[torch.from_numpy(three).to(cuda())] * page
    weaker = torch.from_numpy(weaker).to(cuda())
    before[at + weaker] = before[at + 2]
    assert torch.equal(kv, before) and S.seer_check_device() == 0


def test_far_pages():
    """A pool of more than 2^31 values and 2^32 bytes, its last pages in use."""
    rng = np.random.default_rng(0)
    hq, hk, dh, page = 8, 8, 128, 64
    n_pages = 17000                               # 1088000 rows of 2048 values, 4.46e9 bytes
    kv = torch.empty(n_pages * page, 2 * hk * dh, dtype=torch.bfloat16, device=cuda())
    assert kv.numel() > 2 ** 31
    last = [n_pages - 1, n_pages - 3, n_pages - 2, 0]
    table = i32([last])
    pages = S.make_pages(kv, table, n_pages, page, 4, hk, dh)
    x = rnd(rng, (200, 3 * hk * dh), "bf16")
    slot = i32([last[t // page] * page + t % page for t in range(200)])
    rot, rate = rotary(10000.0, 64, True, "none")
    qk = torch.zeros(200, 2 * hk * dh, dtype=torch.bfloat16, device=cuda())
    S.seer_kv_append_rotary(x, x.stride(0), "bf16", hq, 200, None, slot, i32(range(200)), None, None, 0, rot, qk, qk.stride(0), pages)
    stored = kv[slot.long()]
    assert torch.equal(stored[:, :hk * dh], qk[:, hq * dh:]) and torch.equal(stored[:, hk * dh:], x[:, 2 * hk * dh:])
    s = dict(kv=kv, table=np.array([last]), q=qk[:, :hq * dh], kv_len=[200], cu=[0, 200], n_pages=n_pages, max_pages=4, ld=200)
    mass_in = torch.zeros(1, 200, device=cuda())
    keys = host(stored)[:, :hk * dh].reshape(200, hk, dh)
    for window in (1, 30):
        out, _ = run_mass(s, "bf16", hq, hk, dh, page, window, 0.0, mass_in, None)
        look = list(range(200 - window, 200))
        (w, err), = R.mass(host(qk[:, :hq * dh]).reshape(200, hq, dh), keys, [[0]], 1 << 30, [(look, look, 200, 200)], 0.0, host(mass_in), dh)
        close(out[0], w, err, "mass")
    before = kv[slot.long()].clone()
    S.seer_kv_evict("bf16", i32([200]), i32([2]), i32([[198, 199]]), i32([[0, 70]]), 2, 1, pages, None, None, 0)
    before[0], before[70] = before[198], before[199]
    assert torch.equal(kv[slot.long()], before) and S.seer_check_device() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("inter,rd", [(True, 12), (True, 20), (False, 12), (True, 2)])
def test_what_does_not_turn_keeps_its_bits(dt, inter, rd):
    raw = {"f32": torch.int32, "bf16": torch.int16, "f16": torch.int16}[dt]
    gen = torch.Generator(device=cuda()).manual_seed(3)
    info = torch.iinfo(raw)
    bits = torch.randint(info.min, info.max, (64, 96), device=cuda(), generator=gen, dtype=raw)      # NaNs of every kind among them
    x = bits.view(TDT[dt])
    rot, _ = rotary(10000.0, rd, inter, "none")
    out = torch.zeros_like(x)
    S.seer_rotate(x, 96, dt, 2, 48, 64, None, i32(range(64)), rot, out, 96)
    heads, got = bits.view(64, 2, 48), out.view(raw).view(64, 2, 48)
    assert torch.equal(got[..., rd:], heads[..., rd:])
    S.seer_rotate(x, 96, dt, 2, 48, 64, None, i32(range(64)), rot, x, 96)
    assert torch.equal(x.view(raw).view(64, 2, 48)[..., rd:], got[..., rd:])


def test_append_rotary_counts_rows_on_the_device():
    rng = np.random.default_rng(5)
    x = rnd(rng, (40, 4 * 64), "bf16")
    kv, table = torch.zeros(64, 2 * 64, dtype=torch.bfloat16, device=cuda()), i32([[0]])
    pages = S.make_pages(kv, table, 8, 8, 1, 1, 64)
    rot, _ = rotary(10000.0, 64, False, "none")
    out = torch.full((40, 3 * 64), 5.0, dtype=torch.bfloat16, device=cuda())
    S.seer_kv_append_rotary(x, 256, "bf16", 2, 40, i32([7]), i32(range(40)), i32(range(40)), i32([0, 3, 7]), i32([1000, 5]), 2, rot, out, 192, pages)
    assert (out[7:] == 5).all() and (kv[7:] == 0).all() and not (out[:7] == 5).all(1).any()
    S.seer_kv_append_rotary(x, 256, "bf16", 2, 40, None, i32([64] + [-5] + [-1] * 38), i32(range(40)), None, None, 0, rot, None, 0, pages)
    assert S.seer_check_device() == 2 and (kv[7:] == 0).all()


def test_a_wild_offset_costs_its_own_requests_alone():
    rng = np.random.default_rng(6)
    for dt, window in (("f32", 2), ("bf16", 2), ("bf16", 20)):
        s = setup_mass(rng, dt, 4, 2, 64, 16, [40, 50, 60, 70], [2, 2, 2, 2])
        mass_in = torch.rand(4, s["ld"], device=cuda())
        want, _ = run_mass(s, dt, 4, 2, 64, 16, window, 1.0, mass_in, None)
        for bad in (-2 ** 31, 2 ** 31 - 1, -1):
            s["cu"] = np.array([0, 2, bad, 6, 8])
            got, _ = run_mass(s, dt, 4, 2, 64, 16, window, 1.0, mass_in, None)
            assert torch.equal(got[[0, 3]], want[[0, 3]]) and (got[[1, 2]] == -3).all() and S.seer_check_device() == 2
        s["cu"] = np.array([0, 2, 4, 6, 8])


@pytest.mark.parametrize("L,budget", [(16385, 9000), (40000, 1), (40000, 39999), (33000, 32768), (300000, 100000)])
def test_select_over_the_border_of_a_ctas_memory(L, budget):
    """Requests in one CTA's and several CTAs' stretches, and past the keys that they hold."""
    rng = np.random.default_rng(L)
    mass = rng.integers(0, 1000, (1, L)).astype(np.float32)       # ties everywhere
    birth = rng.permutation(L)[None]
    ld_move = max(1, min(budget, L - budget))
    out = [i32([0]) for _ in range(3)] + [torch.full((1, ld_move), -7, dtype=torch.int32, device=cuda()) for _ in range(2)]
    S.seer_evict_select(torch.from_numpy(mass).to(cuda()), i32(birth), L, i32([L]), i32([5]), i32([budget]), 1, 3, 100, *out, ld_move)
    k, g, src, to = R.select(mass[0], birth[0], L, 5, budget, 3, 100)
    assert (int(out[0]), int(out[1]), int(out[2])) == (k, g, len(src))
    assert out[3][0, :len(src)].tolist() == src and out[4][0, :len(to)].tolist() == to


def test_select_of_many_long_requests():
    """More CTAs' worth of rows than the GPU has room for: one CTA a request, rows past its memory."""
    rng = np.random.default_rng(1)
    B, L = 310, 20000
    mass = rng.standard_normal((B, L)).astype(np.float32)
    birth = np.tile(np.arange(L), (B, 1))
    out = [i32([0] * B) for _ in range(3)] + [torch.full((B, 900), -7, dtype=torch.int32, device=cuda()) for _ in range(2)]
    kv_len, budget = rng.integers(19000, L + 1, B), rng.integers(1, 900, B)
    S.seer_evict_select(torch.from_numpy(mass).to(cuda()), i32(birth), L, i32(kv_len), None, i32(budget), B, 0, 50, *out, 900)
    for b in rng.integers(0, B, 12):
        k, g, src, to = R.select(mass[b], birth[b], int(kv_len[b]), 0, int(budget[b]), 0, 50)
        assert (int(out[0][b]), int(out[1][b]), int(out[2][b])) == (k, g, len(src))
        assert out[3][b, :len(src)].tolist() == src and out[4][b, :len(to)].tolist() == to


def test_select_of_the_longest_request():
    """2^31 - 1025 rows, all but five of one weight: indexes next to the end of 32 bits."""
    L = 2 ** 31 - 1025
    mass = torch.ones(1, L, device=cuda())
    gaps = [7, 10 ** 9, 2 ** 31 - 2000, L - 2, L - 1]
    mass[0, gaps] = 0.25
    birth = torch.arange(L, dtype=torch.int32, device=cuda())
    out = [i32([0]) for _ in range(3)] + [torch.full((1, 5), -7, dtype=torch.int32, device=cuda()) for _ in range(2)]
    S.seer_evict_select(mass, birth, L, i32([L]), None, i32([L - 5]), 1, 0, 0, *out, 5)
    assert (int(out[0]), int(out[1]), int(out[2])) == (L - 5, 5, 3) and S.seer_check_device() == 0
    assert out[3][0].tolist() == [L - 5, L - 4, L - 3, -7, -7] and out[4][0].tolist() == gaps[:3] + [-7, -7]


@pytest.mark.parametrize("scaling", ["linear", "turns", "pairs"])
def test_scaled_rates_to_the_last_position(scaling):
    """Far positions of every scaling, in fp32, against angles reduced in integers."""
    rng = np.random.default_rng(8)
    rot, rate = rotary(500000.0, 128, False, scaling, 1.25)
    pos = np.concatenate([rng.integers(0, 2 ** 20, 40), [2 ** 29, 2 ** 31 - 1, -2 ** 31]])
    x = rnd(rng, (len(pos), 128), "f32")
    out = torch.zeros_like(x)
    S.seer_rotate(x, 128, "f32", 1, 128, len(pos), None, i32(pos), rot, out, 128)
    heads = host(x).reshape(-1, 1, 128)
    ref = R.turn(heads, pos, rate, False, 1.25)
    close(out.reshape(-1, 1, 128), ref, R.turn_bound(heads, ref, pos, 128, False, "f32", 1.25), scaling)


def test_a_turn_and_its_inverse():
    """Negative positions turn back, for either layout: three roundings of fp32 each way."""
    rng = np.random.default_rng(9)
    for inter in (False, True):
        rot, _ = rotary(10000.0, 96, inter, "none")
        x = rnd(rng, (50, 128), "f32")
        pos = rng.integers(1, 100000, 50)
        y, z = torch.zeros_like(x), torch.zeros_like(x)
        S.seer_rotate(x, 128, "f32", 1, 128, 50, None, i32(pos), rot, y, 128)
        S.seer_rotate(y, 128, "f32", 1, 128, 50, None, i32(-pos), rot, z, 128)
        size = float(x.abs().max()) * 2
        assert float((z - x).abs().max()) <= size * (16 * 2.0 ** -24 + 2 * math.pi * 2.0 ** -23)


def test_evict_without_lengths_takes_the_rows_that_the_table_holds():
    rng = np.random.default_rng(2)
    s = setup_mass(rng, "bf16", 1, 1, 64, 8, [30, 9], [0, 0])
    table = i32(s["table"])
    pages = S.make_pages(s["kv"], table, s["n_pages"], 8, s["max_pages"], 1, 64)
    kv = s["kv"].clone()
    S.seer_kv_evict("bf16", None, i32([2, 1]), i32([[29, 31], [15, 0]]), i32([[0, 8], [3, 0]]), 2, 2, pages, None, None, 0)

    def row(b, t):
        return int(s["table"][b][t // 8]) * 8 + t % 8
    for b, f, t in ((0, 29, 0), (0, 31, 8), (1, 15, 3)):   # rows 30 to 31 of a last page are its rows, too
        kv[row(b, t)] = kv[row(b, f)]
    assert torch.equal(s["kv"], kv) and S.seer_check_device() == 0
    S.seer_kv_evict("bf16", None, i32([1, 0]), i32([[32, 0], [0, 0]]), i32([[0, 0], [0, 0]]), 2, 2, pages, None, None, 0)   # past the last page
    assert torch.equal(s["kv"], kv) and S.seer_check_device() == 2


def test_append_rotary_of_keys_alone():
    """No query heads, no rotated output; and queries and keys in place without a cache slot."""
    rng = np.random.default_rng(3)
    rot, rate = rotary(10000.0, 64, True, "linear")
    x = rnd(rng, (9, 4 * 64), "f16")
    kv, table = torch.zeros(16, 4 * 64, dtype=torch.float16, device=cuda()), i32([[0]])
    pages = S.make_pages(kv, table, 2, 8, 1, 2, 64)
    before = x.clone()
    S.seer_kv_append_rotary(x, 256, "f16", 0, 9, None, i32(range(9)), i32(range(100, 109)), i32([0, 9]), i32([50]), 1, rot, None, 0, pages)
    heads = host(before).reshape(9, 4, 64)
    ref = R.turn(heads[:, :2], range(150, 159), rate, True)
    close(kv[:9, :128].reshape(9, 2, 64), ref, R.turn_bound(heads[:, :2], ref, range(150, 159), 64, True, "f16"), "keys")
    assert torch.equal(kv[:9, 128:], before[:, 128:]) and torch.equal(x, before) and (kv[9:] == 0).all()


def test_requests_may_share_pages_that_are_only_read():
    rng = np.random.default_rng(4)
    for dt, hq, window in (("f32", 4, 1), ("bf16", 4, 1), ("bf16", 24, 2)):
        s = setup_mass(rng, dt, hq, 2, 64, 16, [100, 100], [2, 2])
        s["table"][1][:6] = s["table"][0][:6]             # 96 rows of a common prompt
        mass_in = torch.rand(2, s["ld"], device=cuda())
        out, birth = run_mass(s, dt, hq, 2, 64, 16, window, 1.0, mass_in, None)
        check_mass(s, out, birth, dt, hq, 2, 64, 16, window, 1.0, mass_in, None)


def test_results_do_not_depend_on_launch_overlap():
    rng = np.random.default_rng(5)
    for dt, hq, window in (("f32", 4, 2), ("bf16", 4, 2), ("bf16", 24, 2)):
        s = setup_mass(rng, dt, hq, 2, 64, 16, [500, 33, 0], [2, 1, 2])
        mass_in = torch.rand(3, s["ld"], device=cuda())
        results = []
        for overlap in (True, False):
            was = S.seer_set_launch_overlap(overlap)
            try:
                for _ in range(3):                        # calls behind one another share the workspace's memory
                    out, birth = run_mass(s, dt, hq, 2, 64, 16, window, 1.0, mass_in, [1, 2, 3])
                kv, table = s["kv"].clone(), i32(s["table"])
                pages = S.make_pages(kv, table, s["n_pages"], 16, s["max_pages"], 2, 64)
                t = [i32([0] * 3) for _ in range(3)] + [torch.zeros(3, 60, dtype=torch.int32, device=cuda()) for _ in range(2)]
                lens = i32(s["kv_len"])
                S.seer_evict_select(out, birth, s["ld"], lens, i32([1, 2, 3]), i32([450, 20, 2]), 3, 1, 2, *t, 60)
                S.seer_kv_evict(dt, lens, t[2], t[3], t[4], 60, 3, pages, out, birth, s["ld"])
                torch.cuda.synchronize()
            finally:
                S.seer_set_launch_overlap(was)
            results.append([out, birth, kv, *t])
        assert all(torch.equal(a, b) for a, b in zip(*results))
    assert S.seer_check_device() == 0
