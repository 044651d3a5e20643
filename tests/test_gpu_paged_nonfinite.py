"""Infinite and NaN values in the paged cache's attention: they reach the rows that see them,
and only those, however long the prompt or the cache is."""
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


@pytest.mark.parametrize("dt,dh,bad", [("bf16", 128, math.nan), ("f16", 64, math.inf), ("f16", 128, math.nan)])
def test_a_bad_value_late_in_a_long_prompt(dt, dh, bad):
    """40000 rows with one bad value, between two healthy prompts."""
    rng = np.random.default_rng(1)
    hq, hk, lens = 8, 1, [90, 40000, 300]
    T, at, col = sum(lens), 90 + 39900, 5
    x = rnd(rng, (T, (hq + 2 * hk) * dh), dt)
    h = host(x).reshape(T, hq + 2 * hk, dh)
    x[at, (hq + hk) * dh + col] = bad
    o = torch.full((T, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    ld = x.stride(0)
    S.seer_attention_causal(x, ld, x[:, hq * dh:], ld, x[:, (hq + hk) * dh:], ld, o, o.stride(0), dt, i32([0, 90, 40090, T]), 3, T, hq, hk, dh)
    assert S.seer_check_device() in (0, 6)                  # 6: a stored value is not finite
    got = host(o).reshape(T, hq, dh)
    for a, e in ((0, 90), (T - 300, T)):
        ref, bound = R.causal(h[a:e, :hq], h[a:e, hq:hq + 1], h[a:e, hq + 1:], [0, e - a], dt)
        close(got[a:e], ref, bound)
    for row in (90, 4000, at - 130, at - 64, at - 30, at - 1, at, at + 1, at + 20, at + 40, 90 + 39999):
        for head in (0, 7):
            n = row + 1 - 90
            ref, bound = R.attend(h[row, head][None], h[90:row + 1, hq], h[90:row + 1, hq + 1], np.ones((1, n), bool), dt)
            if row < at:
                close(got[row, head], ref[0], bound[0])
            else:
                keep = np.arange(dh) != col
                close(got[row, head][keep], ref[0][keep], bound[0][keep])
                assert not np.isfinite(got[row, head, col]) and (math.isinf(bad) or np.isnan(got[row, head, col]))


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("n", [1, 9])
def test_a_bad_value_behind_long_caches(dt, dh, n):
    """320 requests over one prefix of 20000 rows: about a whole request's keys to a CTA."""
    rng = np.random.default_rng(2)
    hq, hk, page, ctx, B = 8, 1, 64, 20000 - 20, 320
    shared = ctx // page                                    # whole pages of the prefix, then one page of every request's own
    n_pages = shared + B
    kv = rnd(rng, (n_pages * page, 2 * hk * dh), dt)
    table = np.concatenate([np.tile(np.arange(shared), (B, 1)), shared + np.arange(B)[:, None]], 1)
    q = rnd(rng, (B * n, hq * dh), dt)
    kvh = host(kv).reshape(-1, 2, hk, dh)
    slot = lambda b, t: table[b][t // page] * page + t % page
    kv[slot(7, ctx), hk * dh + 3] = math.nan                # the value of request 7's first new row
    table_dev, o = i32(table), torch.full((B * n, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    pages = S.make_pages(kv, table_dev, n_pages, page, table.shape[1], hk, dh)
    size = S.seer_attention_tree_workspace_size(dt, B, hq, hk, dh, n)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=cuda())
    bits = [1 << i for i in range(n)]                       # every new row sees itself alone
    words = torch.tensor(bits * B, dtype=torch.int64, device=cuda())
    S.seer_attention_tree(q, q.stride(0), o, o.stride(0), dt, i32(range(0, B * n + 1, n)), i32([ctx + n] * B), words, B, B * n, hq, n, pages, ws, size)
    assert S.seer_check_device() in (0, 6)
    got, qh = host(o).reshape(B, n, hq, dh), host(q).reshape(B, n, hq, dh)
    for b in (0, 6, 7, 8, 200, B - 1):
        ref, bound = R.tree(qh[b], kvh, [table[b].tolist()], page, [0, n], [ctx + n], bits, dt)
        lost = np.zeros(ref.shape, bool)
        lost[0, :, 3] = b == 7
        assert np.isnan(got[b][lost]).all()
        close(got[b][~lost], ref[~lost], bound[~lost])


@pytest.mark.parametrize("dt,dh", [("bf16", 128), ("f16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("ctx,n,page", [(70, 3, 16), (2600, 3, 64), (2600, 40, 64), (9000, 1, 64)])
@pytest.mark.parametrize("what", ["value", "key", "drafted value", "drafted key"])
def test_paged_rows_that_see_a_nan_are_nan(dt, dh, ctx, n, page, what):
    """A NaN value in its column, a NaN key in every column, of exactly the rows that see it, in requests of one
    piece and of many.  Keys behind the 60th make the cached one's weight e^-200 or less: 0 in 32 bits."""
    rng = np.random.default_rng(ctx + n)
    hq, hk, kv_len = 4, 2, [ctx + n, 33]
    need = [math.ceil(v / page) for v in kv_len]
    order = rng.permutation(sum(need) + 2)
    tab = [order[:need[0]].tolist(), order[need[0]:sum(need)].tolist() + [-1] * (need[0] - need[1])]
    kv = torch.zeros((len(order) * page, 2 * hk * dh), dtype=TDT[dt], device=cuda())
    rows = np.array([tab[0][t // page] * page + t % page for t in range(kv_len[0])])
    keys = torch.zeros((kv_len[0], 2 * hk * dh), dtype=TDT[dt], device=cuda())
    keys[60:, :hk * dh] = 5.0
    keys[:, hk * dh:] = 1.0
    where = ctx if what.startswith("drafted") else 20
    if what.endswith("value"):
        keys[where, (hk + 1) * dh + 1] = math.nan           # column 1 of value head 1: query heads 2 and 3
    else:
        keys[where, dh + 1] = math.nan
    kv[torch.from_numpy(rows).to(cuda())] = keys
    q = torch.full((n + 1, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    bits = [(1 << i) | (i == n - 1) for i in range(n)]      # a row sees itself, the last one row 0 too
    words = torch.tensor(bits + [1], dtype=torch.int64, device=cuda())
    size = S.seer_attention_tree_workspace_size(dt, 2, hq, hk, dh, n)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=cuda())
    table, o = i32(tab), torch.full((n + 1, hq * dh), 5.0, dtype=TDT[dt], device=cuda())
    pages = S.make_pages(kv, table, len(order), page, need[0], hk, dh)
    S.seer_attention_tree(q, q.stride(0), o, o.stride(0), dt, i32([0, n, n + 1]), i32(kv_len), words, 2, n + 1, hq, n, pages, ws, size)
    got = host(o).reshape(n + 1, hq, dh)
    sees = np.array([not what.startswith("drafted") or i == 0 or i == n - 1 for i in range(n)] + [False])
    lost = np.zeros((n + 1, hq, dh), bool)
    lost[sees, 2:, 1] = True
    if what.endswith("key"):
        lost[sees, 2:] = True
    assert np.array_equal(np.isnan(got), lost)
    assert (np.abs(got[:n][~lost[:n]] - 1.0) <= 2.0 ** -7).all() and (got[n] == 0).all()
    S.seer_check_device()
