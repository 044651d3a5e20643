"""Refusals of the entry points that keep a paged cache within a budget, which need no GPU, and their
reference by hand."""
import ctypes
import math

import numpy as np
import pytest
import torch

from tests import budget_reference as R

S = pytest.importorskip("paper_2607_14557_gb300.seer")
P = 1 << 20                       # a 16-byte aligned address that no refused call follows
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_14557_gb300 import build
    build.build()


def pages(**kw):
    a = dict(kv=P, table=P, n_pages=10, page_size=16, max_pages=4, n_kv_heads=2, head_dim=64)
    a.update(kw)
    return S.seer_pages(*a.values())


def rot(**kw):
    a = dict(theta=1e4, rotary_dim=32)
    a.update(kw)
    return ctypes.byref(S.make_rotary(**a))


RAMP = dict(scaling="turns", factor=8.0, low=1.0, high=4.0, original_len=8192)
BAD_ROTARY = [
    (dict(theta=0.5), INVALID), (dict(theta=math.nan), INVALID), (dict(theta=math.inf), INVALID), (dict(rotary_dim=0), INVALID),
    (dict(rotary_dim=33), INVALID), (dict(rotary_dim=66), INVALID), (dict(rotary_dim=-2), INVALID), (dict(rotary_dim=30), UNSUPPORTED),
    (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(interleaved=2), INVALID), (dict(magnitude=math.inf), INVALID),
    (dict(scaling="linear", factor=0.5), INVALID), (dict(scaling="linear", factor=math.nan), INVALID),
    (dict(RAMP, low=0.0), INVALID), (dict(RAMP, low=4.0), INVALID), (dict(RAMP, high=math.inf), INVALID),
    (dict(RAMP, original_len=0), INVALID), (dict(RAMP, factor=math.inf), INVALID), (dict(RAMP, scaling="pairs", theta=1.0), INVALID)]


def rotate(**kw):
    a = dict(x=P, ld=256, dt=1, heads=4, dh=64, T=8, M=None, pos=P, rot=rot(), out=2 * P, ld_out=256, stream=None)
    a.update(kw)
    return S.lib().seer_rotate(*a.values())


def append(pg=None, **kw):
    a = dict(qkv=P, ld=512, dt=1, heads=4, T=8, M=None, slot=P, pos=P, cu=P, shift=P, B=2, rot=rot(), rotated=2 * P, ld_rot=384,
             pages=ctypes.byref(pages(**(pg or {}))), stream=None)
    a.update(kw)
    return S.lib().seer_kv_append_rotary(*a.values())


@pytest.mark.parametrize("kw,status", BAD_ROTARY)
def test_rotary_refuses(kw, status):
    assert rotate(rot=rot(**kw)) == status and b"rotate" in S.lib().seer_last_error()
    assert append(rot=rot(**kw)) == status and b"rotary append" in S.lib().seer_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(pos=None), INVALID), (dict(rot=None), INVALID), (dict(dt=4), INVALID),
    (dict(heads=0), INVALID), (dict(dh=0), INVALID), (dict(dh=72), UNSUPPORTED), (dict(dh=256), UNSUPPORTED), (dict(T=-1), INVALID),
    (dict(T=(1 << 30) + 1), UNSUPPORTED), (dict(ld=255), INVALID), (dict(ld=260), UNSUPPORTED), (dict(x=P + 8), UNSUPPORTED),
    (dict(out=P, ld_out=264), INVALID), (dict(ld_out=8), INVALID), (dict(heads=1 << 15, ld=1 << 21, ld_out=1 << 21), UNSUPPORTED)])
def test_rotate_refuses(kw, status):
    assert rotate(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(qkv=None), INVALID), (dict(ld=511), INVALID), (dict(ld=516), UNSUPPORTED), (dict(ld_rot=383), INVALID), (dict(rotated=P), INVALID),
    (dict(slot=None), INVALID), (dict(pos=None), INVALID), (dict(cu=None), INVALID), (dict(B=0), INVALID), (dict(T=-1), INVALID),
    (dict(B=S.MAX_REQUESTS + 1), UNSUPPORTED), (dict(heads=-1), INVALID), (dict(dt=3), INVALID), (dict(pages=None), INVALID),
    (dict(pg=dict(page_size=12)), UNSUPPORTED), (dict(pg=dict(kv=None)), INVALID)])
def test_append_rotary_refuses(kw, status):
    assert append(**kw) == status


def mass(pg=None, **kw):
    a = dict(q=P, ld=256, dt=1, cu=P, kv=P, acc=None, n_acc=None, draft=0, window=4, B=2, T=8, T_kv=100, hq=4,
             pages=ctypes.byref(pages(**(pg or {}))), keep=1.0, gone=None, mass_in=P, mass_out=2 * P, birth=P, ld_mass=64, ws=P, ws_bytes=0,
             stream=None)
    a.update(kw)
    return S.lib().seer_attention_mass(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(ld=255), INVALID), (dict(ld=260), UNSUPPORTED), (dict(dt=5), INVALID), (dict(cu=None), INVALID),
    (dict(kv=None), INVALID), (dict(acc=P), INVALID), (dict(n_acc=P), INVALID), (dict(acc=P, n_acc=P, draft=0), INVALID),
    (dict(acc=P, n_acc=P, draft=65), INVALID), (dict(window=0), INVALID), (dict(window=65), INVALID), (dict(B=0), INVALID),
    (dict(B=S.MAX_REQUESTS + 1), UNSUPPORTED), (dict(T=-1), INVALID), (dict(T_kv=-1), INVALID), (dict(hq=3), INVALID),
    (dict(keep=math.nan), INVALID), (dict(mass_in=None), INVALID), (dict(mass_out=None), INVALID), (dict(ld_mass=0), INVALID),
    (dict(pg=dict(head_dim=80)), UNSUPPORTED), (dict(pg=dict(table=None)), INVALID), (dict(pages=None), INVALID),
    (dict(dt=0, hq=1026, ld=1026 * 64, window=16), UNSUPPORTED), (dict(B=16384, T_kv=2 ** 31 - 1, window=64, hq=128, ld=8192), UNSUPPORTED)])
def test_mass_refuses(kw, status):
    assert mass(**kw) == status


@pytest.mark.parametrize("args,status", [((1, 0, 10, 4, 2, 64, 8), INVALID), ((1, 2, -1, 4, 2, 64, 8), INVALID), ((1, 2, 10, 5, 2, 64, 8), INVALID),
                                         ((1, 2, 10, 4, 2, 80, 8), UNSUPPORTED), ((1, 2, 10, 4, 2, 64, 0), INVALID),
                                         ((1, 2, 10, 4, 2, 64, 65), INVALID), ((9, 2, 10, 4, 2, 64, 8), INVALID)])
def test_mass_workspace_refuses(args, status):
    out = ctypes.c_size_t(0)
    assert S.lib().seer_attention_mass_workspace_size(*args, ctypes.byref(out)) == status


def select(**kw):
    a = dict(mass=P, birth=2 * P, ld=64, kv=3 * P, gone=4 * P, budget=5 * P, B=2, sinks=0, recent=0, len=6 * P, gone_out=7 * P, n=8 * P,
             src=9 * P, to=10 * P, ld_move=8, stream=None)
    a.update(kw)
    return S.lib().seer_evict_select(*a.values())


@pytest.mark.parametrize("kw,status", [
    *((dict([(k, None)]), INVALID) for k in ("mass", "birth", "kv", "budget", "len", "gone_out", "n", "src", "to")),
    (dict(B=0), INVALID), (dict(B=S.MAX_REQUESTS + 1), UNSUPPORTED), (dict(ld=0), INVALID), (dict(ld=2 ** 31 - 1), UNSUPPORTED),
    (dict(ld_move=0), INVALID), (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID), (dict(n=3 * P), INVALID), (dict(len=4 * P), INVALID),
    (dict(gone_out=3 * P), INVALID), (dict(src=P), INVALID), (dict(to=2 * P), INVALID), (dict(len=5 * P), INVALID), (dict(src=10 * P), INVALID)])
def test_select_refuses(kw, status):
    assert select(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=3), INVALID), (dict(n=None), INVALID), (dict(src=None), INVALID), (dict(to=None), INVALID), (dict(ld_move=0), INVALID),
    (dict(B=0), INVALID), (dict(ld=0), INVALID), (dict(mass=None, ld=-1), INVALID), (dict(pages=None), INVALID)])
def test_evict_refuses(kw, status):
    a = dict(dt=1, kv=P, n=P, src=P, to=P, ld_move=4, B=2, pages=ctypes.byref(pages()), mass=P, birth=P, ld=8, stream=None)
    a.update(kw)
    assert S.lib().seer_kv_evict(*a.values()) == status


def test_calls_for_no_rows_take_buffers_without_an_address():
    for dt in (0, 1, 2):
        assert rotate(dt=dt, T=0, x=None, out=None, pos=None, ld=0, ld_out=0) == 0
        assert append(dt=dt, T=0, qkv=None, slot=None, pos=None, rotated=None, ld=0, ld_rot=0) == 0
    assert rotate(T=0, rot=rot(theta=0.0)) == INVALID and append(T=0, rot=rot(theta=0.0)) == INVALID


# ------------------------------------------------------------------ what tensors have to hold
BF, F32 = torch.bfloat16, torch.float32
B, T, HQ, HK, DH, LD = 2, 8, 4, 2, 64, 20


def ints(n):
    return torch.zeros(n, dtype=torch.int32)


def pool(dtype=BF, requests=B):
    return S.make_pages(torch.zeros((160, 2 * HK * DH), dtype=dtype), torch.zeros((requests, 4), dtype=torch.int32), 10, 16, 4, HK, DH)


def t_rotate(**kw):
    a = dict(x=torch.zeros(T, 256, dtype=BF), ld=256, dt="bf16", heads=4, dh=64, T=T, M=ints(1), pos=ints(T), rot=S.make_rotary(1e4, 64),
             out=torch.zeros(T, 256, dtype=BF), ld_out=256)
    a.update(kw)
    S.seer_rotate(*a.values())


def t_append(**kw):
    a = dict(qkv=torch.zeros(T, 512, dtype=BF), ld=512, dt="bf16", heads=HQ, T=T, M=None, slot=ints(T), pos=ints(T), cu=ints(B + 1), shift=ints(B),
             B=B, rot=S.make_rotary(1e4, 64), rotated=torch.zeros(T, 384, dtype=BF), ld_rot=384, pages=pool())
    a.update(kw)
    S.seer_kv_append_rotary(*a.values())


def t_mass(**kw):
    a = dict(q=torch.zeros(T, 256, dtype=BF), ld=256, dt="bf16", cu=ints(B + 1), kv=ints(B), acc=ints(B * 5), n_acc=ints(B), draft=5, window=4, B=B,
             T=T, T_kv=100, hq=HQ, pages=pool(), keep=1.0, gone=ints(B), mass_in=torch.zeros(B, LD), mass_out=torch.zeros(B, LD), birth=ints(B * LD),
             ld_mass=LD, ws=torch.zeros(64, dtype=torch.uint8), ws_bytes=64)
    a.update(kw)
    S.seer_attention_mass(*a.values())


def t_select(**kw):
    a = dict(mass=torch.zeros(B, LD), birth=ints(B * LD), ld=LD, kv=ints(B), gone=ints(B), budget=ints(B), B=B, sinks=0, recent=0, len=ints(B),
             gone_out=ints(B), n=ints(B), src=ints(B * 6), to=ints(B * 6), ld_move=6)
    a.update(kw)
    S.seer_evict_select(*a.values())


def t_evict(**kw):
    a = dict(dt="bf16", kv=ints(B), n=ints(B), src=ints(B * 6), to=ints(B * 6), ld_move=6, B=B, pages=pool(), mass=torch.zeros(B, LD),
             birth=ints(B * LD), ld=LD)
    a.update(kw)
    S.seer_kv_evict(*a.values())


HELD = [
    (t_rotate, dict(x=torch.zeros(T, 256)), "x is"), (t_rotate, dict(T=T + 1), "x:"), (t_rotate, dict(out=torch.zeros(T - 1, 256, dtype=BF)), "out:"),
    (t_rotate, dict(pos=ints(T - 1)), "position"), (t_rotate, dict(M=ints(0)), "M_dev"), (t_rotate, dict(rot=b"short"), "rotary"),
    (t_append, dict(qkv=torch.zeros(T, 511, dtype=BF)), "qkv"), (t_append, dict(rotated=torch.zeros(T, 383, dtype=BF)), "rotated"),
    (t_append, dict(slot=ints(T - 1)), "slot"), (t_append, dict(pos=ints(T - 1)), "position"), (t_append, dict(cu=ints(B)), "cu_new"),
    (t_append, dict(shift=ints(B - 1)), "shift"), (t_append, dict(pages=pool(F32)), "pool"),
    (t_mass, dict(q=torch.zeros(T, 256)), "q is"), (t_mass, dict(cu=ints(B)), "cu_new"), (t_mass, dict(kv=ints(1)), "kv_len"),
    (t_mass, dict(acc=ints(9)), "accepted"), (t_mass, dict(n_acc=ints(1)), "n_accepted"), (t_mass, dict(gone=ints(1)), "gone"),
    (t_mass, dict(mass_in=torch.zeros(B, LD - 1)), "mass_in"), (t_mass, dict(mass_out=torch.zeros(B, LD - 1)), "mass_out"),
    (t_mass, dict(birth=ints(B * LD - 1)), "birth"), (t_mass, dict(ws_bytes=65), "ws"), (t_mass, dict(pages=pool(requests=1)), "table"),
    (t_select, dict(mass=torch.zeros(B, LD - 1)), "mass"), (t_select, dict(birth=ints(1)), "birth"), (t_select, dict(kv=ints(1)), "kv_len"),
    (t_select, dict(gone=ints(1)), "gone"), (t_select, dict(budget=ints(1)), "budget"), (t_select, dict(len=ints(1)), "len_out"),
    (t_select, dict(gone_out=ints(1)), "gone_out"), (t_select, dict(n=ints(1)), "n_moves"), (t_select, dict(src=ints(11)), "move_from"),
    (t_select, dict(to=ints(11)), "move_to"),
    (t_evict, dict(kv=ints(1)), "kv_len"), (t_evict, dict(n=ints(1)), "n_moves"), (t_evict, dict(src=ints(11)), "move_from"),
    (t_evict, dict(to=ints(11)), "move_to"), (t_evict, dict(mass=torch.zeros(1, LD)), "mass"), (t_evict, dict(birth=ints(LD)), "birth"),
    (t_evict, dict(pages=pool(F32)), "pool"), (t_evict, dict(pages=pool(requests=1)), "table")]


@pytest.mark.parametrize("i", range(len(HELD)))
def test_calls_refuse_tensors_that_do_not_hold_what_they_name(i):
    call, kw, name = HELD[i]
    with pytest.raises(ValueError, match=name):
        call(**kw)


@pytest.mark.parametrize("call", [t_rotate, t_append, t_mass, t_select, t_evict])
def test_whole_tensors_go_on_to_the_device_check(call):
    if torch.cuda.is_available():
        with pytest.raises(ValueError, match="device"):
            call()
    else:
        with pytest.raises(RuntimeError):                   # no device to compare with
            call()


# ------------------------------------------------------------------ the reference, by hand
def test_reference_rates_by_hand():
    assert np.allclose(R.rates(100.0, 4), [1.0, 0.1])
    assert np.allclose(R.rates(100.0, 4, "linear", 4.0), [0.25, 0.025])
    # 628.3 positions: 100 turns of the first pair, 10 of the second
    n = 200 * math.pi
    assert np.allclose(R.rates(100.0, 4, "turns", 4.0, 5.0, 15.0, n), [1.0, 0.1 * (0.5 + 0.5 / 4)])
    assert np.allclose(R.rates(100.0, 4, "turns", 4.0, 20.0, 90.0, n), [1.0, 0.025])
    # pair i makes 10^(2 - i) turns: 99 a little behind pair 0, 1.1 a little before pair 2; the ramp from 0 to 2
    assert np.allclose(R.rates(100.0, 4, "pairs", 4.0, 1.1, 99.0, n), [1.0, 0.1 * (1 / 2 + 1 / 2 / 4)])


def test_reference_turn_by_hand():
    x = np.arange(12.0).reshape(1, 1, 12)
    for inter, pairs in ((False, [(0, 2), (1, 3)]), (True, [(0, 1), (2, 3)])):
        y = R.turn(x, [3], [0.5, 0.01], inter, 2.0)
        for (a, b), r in zip(pairs, (0.5, 0.01)):
            c, s = math.cos(3 * r), math.sin(3 * r)
            assert np.allclose([y[0, 0, a], y[0, 0, b]], [2 * (a * c - b * s), 2 * (b * c + a * s)])
        assert np.allclose(y[0, 0, 4:], x[0, 0, 4:])


def test_reference_mass_by_hand():
    # equal keys: the row at place i of n = 2 new rows behind one cached row sees 2 + i rows alike
    (w, _), = R.mass(np.ones((2, 2, 4)), np.ones((8, 1, 4)), [[0]], 8, [([0, 1], [0, 1], 2, 3)], 0.5, [[4.0, 9.0, 9.0]], 4)
    assert np.allclose(w, [2 + 2 * (1 / 2 + 1 / 3), 2 * (1 / 2 + 1 / 3), 2 / 3])


def test_reference_select_by_hand():
    mass, birth = [0.5, 3.0, math.nan, 3.0, 0.1, 9.0], [0, 1, 2, 3, 4, 5]
    assert R.select(mass, birth, 6, 0, 3, 0, 0) == (3, 3, [5], [0])
    assert R.select(mass, birth, 6, 0, 3, 1, 2) == (3, 3, [4, 5], [1, 2])
    assert R.select(mass, [7, 1, 2, 3, 4, 0], 6, 3, 2, 1, 3) == (2, 7, [5], [1])
