"""What the paged cache's entry points promise about calls that are odd, but allowed."""
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


def rnd(rng, shape, dt):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TDT[dt]).to(cuda())


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound):
    bad = ~(np.abs(got - ref) <= bound + 1e-30)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4])


@pytest.mark.parametrize("dt,dh", [("f32", 64), ("f32", 128), ("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("cu,good", [
    ([0, 100, 2 ** 31 - 1, 200, 300], [(0, 100), (200, 300)]), ([0, 60, 40, 300], [(0, 40)]), ([-5, 40, 300], [(40, 300)]),
    ([0, 100, 301], [(0, 100)]), ([0, 300, 100, 400], [(0, 300)]), ([300, 0, 300], [(0, 300)]), ([5, 0, 0], []), ([100, 200, 0, 50], [(100, 200), (0, 50)]),
    ([0] + [10 * i for i in range(1, 25)] + [-1] + [250 + i for i in range(50)] + [300], [(0, 240), (250, 300)])])
def test_causal_offsets_that_fall_cost_their_own_rows_alone(dt, dh, cu, good):
    """good: rows of sequences that lie in the buffers, as far as no other such sequence has them too."""
    rng = np.random.default_rng(3)
    hq, hk, T, B = 8, 1, 300, len(cu) - 1
    x = rnd(rng, (T, (hq + 2 * hk) * dh), dt)
    h = host(x).reshape(T, hq + 2 * hk, dh)
    o = torch.full((T, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    ld = x.stride(0)
    S.seer_attention_causal(x, ld, x[:, hq * dh:], ld, x[:, (hq + hk) * dh:], ld, o, o.stride(0), dt, i32(cu), B, T, hq, hk, dh)
    assert S.seer_check_device() == 2
    got = host(o).reshape(T, hq, dh)
    taken = [(a, e) for a, e in zip(cu[:-1], cu[1:]) if 0 <= a <= e <= T]
    for a, e in taken:
        rows = [r for r in range(a, e) if any(lo <= r < hi for lo, hi in good)]
        if rows:
            ref, bound = R.causal(h[a:e, :hq], h[a:e, hq:hq + hk], h[a:e, hq + hk:], [0, e - a], dt)
            at = np.array(rows) - a
            close(got[a:e][at], ref[at], bound[at])
    free = np.ones(T, bool)                                 # rows of no sequence are as they were
    for a, e in taken:
        free[a:e] = False
    assert (got[free] == 5.0).all()


@pytest.mark.parametrize("dt,dh", [("f32", 64), ("bf16", 128), ("f16", 64)])
def test_offsets_and_lengths_of_minus_2_31(dt, dh):
    """The difference to an offset of -2^31 passes 2^31: it is inconsistent like any other."""
    rng = np.random.default_rng(6)
    hq, hk, T, cu = 8, 1, 300, [0, 7, -2 ** 31, 9, 9, 300]
    x = rnd(rng, (T, (hq + 2 * hk) * dh), dt)
    h = host(x).reshape(T, hq + 2 * hk, dh)
    o = torch.full((T, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    ld = x.stride(0)
    S.seer_attention_causal(x, ld, x[:, hq * dh:], ld, x[:, (hq + hk) * dh:], ld, o, o.stride(0), dt, i32(cu), 5, T, hq, hk, dh)
    assert S.seer_check_device() == 2
    got = host(o).reshape(T, hq, dh)
    for a, e in ((0, 7), (9, 300)):
        ref, bound = R.causal(h[a:e, :hq], h[a:e, hq:hq + hk], h[a:e, hq + hk:], [0, e - a], dt)
        close(got[a:e], ref, bound)
    assert (got[7:9] == 5.0).all()
    # the same over pages: requests 0, 3 and 4 are well
    page, kv_len, cu = 16, [40, 9, -2 ** 31, 30, 25], [0, 2, -2 ** 31, 4, 5, 8]
    tab = np.arange(15).reshape(5, 3)
    kv = rnd(rng, (15 * page, 2 * hk * dh), dt)
    table, q = i32(tab), x[:8, :hq * dh].contiguous()
    pages = S.make_pages(kv, table, 15, page, 3, hk, dh)
    size = S.seer_attention_tree_workspace_size(dt, 5, hq, hk, dh, 4)
    ws, o = torch.full((size,), 255, dtype=torch.uint8, device=cuda()), torch.full((8, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    S.seer_attention_tree(q, q.stride(0), o, o.stride(0), dt, i32(cu), i32(kv_len), None, 5, 8, hq, 4, pages, ws, size)
    assert S.seer_check_device() == 2
    got, kvh = host(o).reshape(8, hq, dh), host(kv).reshape(-1, 2, hk, dh)
    for b, a, e in ((0, 0, 2), (3, 4, 5), (4, 5, 8)):
        ref, bound = R.tree(host(q).reshape(8, hq, dh)[a:e], kvh, [tab[b].tolist()], page, [0, e - a], [kv_len[b]], None, dt)
        close(got[a:e], ref, bound)
    assert (got[2:4] == 5.0).all()


def test_accept_past_the_longest_request_keeps_nothing():
    """A request has at most 2^31 - 1025 rows, so that the lengths after it are still lengths."""
    kv, table = torch.zeros((5 * 1024, 128), dtype=torch.bfloat16, device=cuda()), torch.zeros((3, 1 << 21), dtype=torch.int32, device=cuda())
    pages = S.make_pages(kv, table, 5, 1024, 1 << 21, 1, 64)
    top = 2 ** 31 - 1025
    for cached, code, want in (([top - 2, 7, 8], 0, [top, 9, 10]), ([top - 1, 7, 8], 2, [top - 1, 9, 10]), ([2 ** 31 - 1024 + 1000, 7, 8], 2, [2 ** 31 - 24, 9, 10])):
        out = i32([-7] * 3)
        S.seer_kv_accept("bf16", i32(cached), i32([[0, 1]] * 3), i32([2] * 3), 3, 2, pages, out)
        assert S.seer_check_device() == code and out.tolist() == want


def test_steps_without_rows():
    """Empty tensors have no address; a step that adds no row calls with them all the same."""
    B, page, hq, hk, dh = 2, 16, 4, 2, 64
    kv, table = rnd(np.random.default_rng(0), (10 * page, 2 * hk * dh), "bf16"), i32([[0, 1], [2, 3]])
    before = kv.clone()
    pages = S.make_pages(kv, table, 10, page, 2, hk, dh)
    none = torch.zeros(0, dtype=torch.int32, device=cuda())
    x, o = torch.zeros((0, (hq + 2 * hk) * dh), dtype=torch.bfloat16, device=cuda()), torch.zeros((0, hq * dh), dtype=torch.bfloat16, device=cuda())
    ld = (hq + 2 * hk) * dh
    cu, kv_len, head_out = i32([-7] * 3), i32([-7] * 2), i32([-7])
    S.seer_page_tables(i32([20, 5]), i32([0, 0]), B, page, 10, none, 0, i32([0]), table, 2, 0, None, cu, kv_len, none, none, None, head_out)
    S.seer_kv_append(x, ld, "bf16", hq, 0, None, none, none, 10000.0, x, ld, pages)
    S.seer_attention_causal(x, ld, x, ld, x, ld, o, hq * dh, "bf16", cu, B, 0, hq, hk, dh)
    S.seer_attention_tree(x, ld, o, hq * dh, "bf16", cu, kv_len, None, B, 0, hq, 4, pages, None, 0)
    assert cu.tolist() == [0, 0, 0] and kv_len.tolist() == [20, 5] and torch.equal(kv, before) and S.seer_check_device() == 0


def test_pages_of_rejected_rows_put_back_keep_the_pool_from_running_dry():
    """Rounds of drafting 24 rows and keeping 1 to 5: every round leaves one or two pages a request that only
    rejected rows filled.  Put back as seer_kv_accept says, the pool holds for ever; left, it is dry within 20 rounds."""
    rng = np.random.default_rng(4)
    B, page, draft, hk, dh, rounds = 4, 16, 24, 1, 64, 60
    max_pages = (100 + 5 * rounds + draft) // page + 2
    n_pages = B * ((100 + 5 * rounds + draft) // page + 1)
    kv = torch.zeros((n_pages * page, 2 * hk * dh), dtype=torch.bfloat16, device=cuda())
    order = rng.permutation(n_pages)
    tab = np.full((B, max_pages), -1)
    tab[:, :7] = order[:7 * B].reshape(B, 7)
    table, free, head = i32(tab), i32(order), i32([7 * B])
    pages = S.make_pages(kv, table, n_pages, page, max_pages, hk, dh)
    cached, new = i32([100] * B), i32([draft] * B)
    kept_rows = [[] for _ in range(B)]
    taken = 0
    for _ in range(rounds):
        cu, kv_len, slot, pos, head_out, len_out = (torch.zeros(n, dtype=torch.int32, device=cuda()) for n in (B + 1, B, B * draft, B * draft, 1, B))
        S.seer_page_tables(cached, new, B, page, n_pages, free, n_pages, head, table, max_pages, B * draft, None, cu, kv_len, slot, pos, None, head_out)
        taken += int(head_out) - int(head)
        assert (slot >= 0).all() and slot.unique().numel() == B * draft
        x = rnd(rng, (B * draft, 2 * hk * dh), "bf16")
        S.seer_kv_append(x, x.stride(0), "bf16", 0, B * draft, None, slot, None, 0.0, None, 0, pages)
        keep = [sorted(rng.choice(draft, int(rng.integers(1, 6)), replace=False).tolist()) for _ in range(B)]
        S.seer_kv_accept("bf16", cached, i32([k + [-1] * (draft - len(k)) for k in keep]), i32([len(k) for k in keep]), B, draft, pages, len_out)
        for b, k in enumerate(keep):
            kept_rows[b] += [x[b * draft + a] for a in k]
        col = torch.arange(max_pages, device=cuda())[None]
        back = (col >= ((len_out + page - 1) // page)[:, None]) & (col < ((kv_len + page - 1) // page)[:, None])
        k = int(back.sum())
        free[int(head_out) - k:int(head_out)] = table[back]
        head.copy_(head_out - k)
        cached.copy_(len_out)
        owned = table[col < ((cached + page - 1) // page)[:, None]].tolist() + free[int(head):].tolist()
        assert sorted(owned) == list(range(n_pages))        # every page in the table or free, once
    assert taken > 2 * n_pages and S.seer_check_device() == 0
    for b in range(B):
        t = torch.arange(100, int(cached[b]), device=cuda())
        rows = table[b].long()[t // page] * page + t % page
        assert torch.equal(kv[rows], torch.stack(kept_rows[b]))


@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1.0])
@pytest.mark.parametrize("top", [2 ** 24, 2 ** 29, 2 ** 31 - 1])
def test_rotation_of_far_positions_against_a_longer_arithmetic(theta, top):
    """Angles in 60 decimal digits.  Counted: fp32 sine and cosine of an angle rounded to fp32 in half turns (2^-25
    of half a turn: pi 2^-25), their 2^-23 each and the products' and sum's 2^-24; the rate's fp64 rounding
    (3.4 2^-53 of it: exp2, its argument, 2 pi, the division) times the position."""
    from decimal import Decimal as D, getcontext
    getcontext().prec = 60
    two_pi = D("6.28318530717958647692528676655900576839433879875021164194988918")
    rng = np.random.default_rng(5)
    dh, T, page = 128, 16, 16
    pos = [top - int(v) for v in rng.integers(0, top // 2, T - 1)] + [top]
    kv, x = torch.zeros((page, 2 * dh), device=cuda()), rnd(rng, (T, 3 * dh), "f32")
    pages = S.make_pages(kv, i32([[0]]), 1, page, 1, 1, dh)
    out = torch.zeros((T, 2 * dh), device=cuda())
    S.seer_kv_append(x, 3 * dh, "f32", 1, T, None, i32(range(T)), i32(pos), theta, out, 2 * dh, pages)
    rate = [D(theta) ** (D(-2 * i) / dh) for i in range(dh // 2)]
    angle = np.array([[float((D(p) * r) % two_pi) for r in rate] for p in pos])
    h, got = host(x)[:, :2 * dh].reshape(T, 2, 2, dh // 2), host(out).reshape(T, 2, 2, dh // 2)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = h[:, :, 0], h[:, :, 1]
    ref = np.stack([a * c - b * s, b * c + a * s], 2)
    bound = (np.abs(a) + np.abs(b))[:, :, None] * (math.pi * 2.0 ** -25 + top * 3.4 * 2.0 ** -53 + 2.0 ** -23 + 3 * 2.0 ** -24)
    close(got, ref, bound)
    assert S.seer_check_device() == 0
