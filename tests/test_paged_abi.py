"""Refusals of the paged cache entry points that need no GPU, and the reference itself."""
import ctypes
import math

import numpy as np
import pytest

from tests import paged_reference as R

S = pytest.importorskip("paper_2607_14557_gb300.seer")
P = 1 << 20                       # a 16-byte aligned address that no refused call follows
INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2607_14557_gb300 import build
    build.build()
    return S.lib()


def pages(**kw):
    a = dict(kv=P, table=P, n_pages=10, page_size=16, max_pages=4, n_kv_heads=2, head_dim=64)
    a.update(kw)
    return S.seer_pages(*a.values())


def tables(L, **kw):
    a = dict(cached=P, new=2 * P, B=2, page=16, n_pages=10, free=P, n_free=4, head=P, table=P, max_pages=4, T=8, parent=None,
             cu=3 * P, kv=4 * P, slot=P, pos=P, mask=None, head_out=2 * P, stream=None)
    a.update(kw)
    return L.seer_page_tables(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(B=-1), INVALID), (dict(B=S.MAX_REQUESTS + 1), UNSUPPORTED), (dict(page=4), UNSUPPORTED),
    (dict(page=24), UNSUPPORTED), (dict(page=2048), UNSUPPORTED), (dict(cached=None), INVALID), (dict(new=None), INVALID),
    (dict(head=None), INVALID), (dict(table=None), INVALID), (dict(cu=None), INVALID), (dict(kv=None), INVALID),
    (dict(slot=None), INVALID), (dict(pos=None), INVALID), (dict(head_out=None), INVALID), (dict(free=None), INVALID),
    (dict(n_free=-1), INVALID), (dict(T=-1), INVALID), (dict(max_pages=0), INVALID), (dict(n_pages=0), INVALID),
    (dict(n_pages=1 << 28), UNSUPPORTED), (dict(head_out=P), INVALID), (dict(kv=P), INVALID), (dict(kv=2 * P), INVALID),
    (dict(cu=2 * P), INVALID), (dict(cu=P), INVALID)])
def test_page_tables_refuse(L, kw, status):
    assert tables(L, **kw) == status and b"page tables" in L.seer_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(T=(1 << 30) + 1), UNSUPPORTED), (dict(mask=64 * P + 4), UNSUPPORTED), (dict(slot=16 * P), INVALID), (dict(pos=16 * P), INVALID),
    (dict(mask=16 * P), INVALID), (dict(table=8 * P), INVALID), (dict(slot=9 * P), INVALID)])
def test_page_tables_refuse_sizes_and_shared_buffers(L, kw, status):
    a = dict(free=8 * P, head=9 * P, table=10 * P, slot=11 * P, pos=12 * P, parent=16 * P)
    a.update(kw)
    assert tables(L, **a) == status and b"page tables" in L.seer_last_error()


def append(L, pg=None, **kw):
    a = dict(qkv=P, ld=4 * 64 + 4 * 64, dt=1, heads=4, T=8, M=None, slot=P, pos=P, theta=1e4, rot=2 * P, ld_rot=6 * 64)
    a.update(kw)
    return L.seer_kv_append(*a.values(), ctypes.byref(pages(**(pg or {}))), None)


BAD_PAGES = [(dict(kv=None), INVALID), (dict(table=None), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=-1), INVALID),
             (dict(page_size=12), UNSUPPORTED), (dict(n_kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
             (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(kv=P + 8), UNSUPPORTED),
             (dict(n_pages=1 << 27), UNSUPPORTED)]


@pytest.mark.parametrize("pg,status", BAD_PAGES)
def test_append_refuses_pools(L, pg, status):
    assert append(L, pg, ld=8192, ld_rot=8192) == status


@pytest.mark.parametrize("kw,status", [
    (dict(qkv=None), INVALID), (dict(ld=511), INVALID), (dict(ld=516), UNSUPPORTED), (dict(qkv=P + 2), UNSUPPORTED),
    (dict(ld_rot=383), INVALID), (dict(rot=P), INVALID), (dict(slot=None), INVALID), (dict(pos=None), INVALID),
    (dict(theta=-1.0), INVALID), (dict(theta=math.nan), INVALID), (dict(theta=math.inf), INVALID), (dict(T=-1), INVALID),
    (dict(heads=-1), INVALID), (dict(dt=3), INVALID)])
def test_append_refuses(L, kw, status):
    assert append(L, **kw) == status


@pytest.mark.parametrize("kw,status", [(dict(T=(1 << 30) + 1), UNSUPPORTED), (dict(theta=0.5), INVALID), (dict(theta=1e-40), INVALID)])
def test_append_refuses_rows_and_bases(L, kw, status):
    assert append(L, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(cached=None), INVALID), (dict(acc=None), INVALID), (dict(n=None), INVALID),
    (dict(draft=0), INVALID), (dict(draft=65), INVALID), (dict(out=None), INVALID), (dict(out=P), INVALID),
    (dict(dt=7), INVALID)])
def test_accept_refuses(L, kw, status):
    a = dict(dt=1, cached=P, acc=3 * P, n=4 * P, B=2, draft=8)
    a.update({k: v for k, v in kw.items() if k != "out"})
    assert L.seer_kv_accept(*a.values(), ctypes.byref(pages()), kw.get("out", 2 * P), None) == status


def causal(L, **kw):
    a = dict(q=P, ld_q=512, k=2 * P, ld_k=256, v=3 * P, ld_v=256, o=4 * P, ld_o=512, dt=1, cu=P, B=1, T=8, hq=4, hk=2, dh=128)
    a.update(kw)
    return L.seer_attention_causal(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(o=None), INVALID), (dict(cu=None), INVALID),
    (dict(B=0), INVALID), (dict(T=-1), INVALID), (dict(hk=3), INVALID), (dict(hq=0), INVALID), (dict(dh=96), UNSUPPORTED),
    (dict(dh=256), UNSUPPORTED), (dict(dt=0, dh=66), UNSUPPORTED), (dict(ld_q=511), INVALID), (dict(ld_k=260), UNSUPPORTED),
    (dict(ld_v=255), INVALID), (dict(ld_o=8), INVALID), (dict(o=P), INVALID), (dict(o=2 * P), INVALID), (dict(v=P + 4), UNSUPPORTED),
    (dict(dt=9), INVALID), (dict(hq=258, hk=2, ld_q=1 << 16, ld_o=1 << 16), UNSUPPORTED)])
def test_causal_refuses(L, kw, status):
    assert causal(L, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(o=P), INVALID), (dict(cu=None), INVALID), (dict(kv=None), INVALID),
    (dict(B=0), INVALID), (dict(T=-1), INVALID), (dict(hq=3), INVALID), (dict(draft=0), INVALID), (dict(draft=65), INVALID),
    (dict(ld_q=100), INVALID), (dict(dt=5), INVALID)])
def test_tree_refuses(L, kw, status):
    a = dict(q=P, ld_q=256, o=2 * P, ld_o=256, dt=1, cu=P, kv=P, mask=None, B=2, T=8, hq=4, draft=4)
    a.update(kw)
    assert L.seer_attention_tree(*a.values(), ctypes.byref(pages()), P, 1 << 30, None) == status


def test_attention_refuses_row_counts_past_30_bits(L):
    assert causal(L, T=(1 << 30) + 1) == UNSUPPORTED
    assert L.seer_attention_tree(P, 256, 2 * P, 256, 1, P, P, None, 2, (1 << 30) + 1, 4, 4, ctypes.byref(pages()), P, 1 << 30, None) == UNSUPPORTED


@pytest.mark.parametrize("mask,pg", [(P + 4, {}), (None, dict(n_kv_heads=1 << 14, max_pages=(1 << 31) - 1, page_size=1024))])
def test_tree_refuses_odd_masks_and_endless_tables(L, mask, pg):
    hk = pg.get("n_kv_heads", 2)
    st = L.seer_attention_tree(P, hk * 64, 2 * P, hk * 64, 1, P, P, mask, 16384 if pg else 2, 8, hk, 4, ctypes.byref(pages(**pg)), P, 1 << 30, None)
    assert st == UNSUPPORTED and (b"aligned" if mask else b"2^50") in L.seer_last_error()


@pytest.mark.parametrize("args,status", [((1, 0, 4, 2, 64, 8), INVALID), ((1, 2, 5, 2, 64, 8), INVALID), ((1, 2, 4, 2, 80, 8), UNSUPPORTED),
                                         ((1, 2, 4, 2, 64, 0), INVALID), ((1, 2, 4, 2, 64, 65), INVALID), ((9, 2, 4, 2, 64, 8), INVALID)])
def test_workspace_size_refuses(L, args, status):
    out = ctypes.c_size_t(0)
    assert L.seer_attention_tree_workspace_size(*args, ctypes.byref(out)) == status


def test_make_pages_refuses_small_pools():
    import torch
    kv, table = torch.zeros(32, 256), torch.zeros(2, 4, dtype=torch.int32)
    S.make_pages(kv, table, 4, 8, 4, 2, 64)
    with pytest.raises(ValueError):
        S.make_pages(kv, table, 5, 8, 4, 2, 64)
    with pytest.raises(ValueError):
        S.make_pages(kv.t(), table, 4, 8, 4, 2, 64)
    with pytest.raises(ValueError):
        S.make_pages(kv, table.long(), 4, 8, 4, 2, 64)


# ------------------------------------------------------------------ the reference, by hand
def test_reference_tables_by_hand():
    cu, kv, slot, pos, mask, table, head = R.page_tables([7, 0], [3, 9], 8, [5, 2, 9, 4], 1, [[6, -1], [-1, -1]])
    assert cu == [0, 3, 12] and kv == [10, 9] and head == 4
    assert table == [[6, 2], [9, 4]]
    assert slot == [6 * 8 + 7, 16, 17] + list(range(72, 80)) + [32]
    assert pos == [7, 8, 9] + list(range(9)) and mask[:3] == [1, 3, 7]


def test_reference_tree_by_hand():
    _, _, _, pos, mask, _, _ = R.page_tables([4], [5], 16, [], 0, [[0]], [[-1, 0, 0, 1, -1]])
    assert pos == [4, 5, 5, 6, 4] and mask == [0b1, 0b11, 0b101, 0b1011, 0b10000]


def test_reference_rotation_is_a_rotation():
    x = np.random.default_rng(0).standard_normal((3, 2, 8))
    y = R.rotate(x, [0, 1, 5], 100.0)
    assert np.allclose(y[0], x[0])
    assert np.allclose((y ** 2).sum(), (x ** 2).sum())
    c, s = math.cos(5 * 100.0 ** (-2 / 8)), math.sin(5 * 100.0 ** (-2 / 8))
    assert np.allclose(y[2, 0, 1], x[2, 0, 1] * c - x[2, 0, 5] * s)


def test_reference_attention_of_equal_keys_averages_values():
    v = np.arange(8.0).reshape(4, 2)
    o, _ = R.attend(np.ones((2, 2)), np.ones((4, 2)), v, np.array([[1, 1, 0, 0], [0, 0, 0, 0]], bool), "f32")
    assert np.allclose(o, [[1, 2], [0, 0]])
