"""The paged cache's Python calls refuse tensors that do not hold what the call names: before a
device is asked for, so these run without one."""
import pytest
import torch

S = pytest.importorskip("paper_2607_14557_gb300.seer")
BF, F32, F16 = torch.bfloat16, torch.float32, torch.float16
HQ, HK, DH, B, T = 4, 2, 64, 2, 8
W = (HQ + 2 * HK) * DH


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_14557_gb300 import build
    build.build()


def ints(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def pool(dtype=BF, rows=160, requests=B):
    return S.make_pages(torch.zeros((rows, 2 * HK * DH), dtype=dtype), torch.zeros((requests, 4), dtype=torch.int32), 10, 16, 4, HK, DH)


def tables(**kw):
    a = dict(cached=ints(B), new=ints(B), B=B, page=16, n_pages=10, free=ints(4), n_free=4, head=ints(1), table=ints(B * 4), max_pages=4, T=T,
             parent=ints(T), cu=ints(B + 1), kv=ints(B), slot=ints(T), pos=ints(T), mask=ints(T, torch.int64), head_out=ints(1))
    a.update(kw)
    S.seer_page_tables(*a.values())


def append(**kw):
    a = dict(qkv=torch.zeros((T, W), dtype=BF), ld=W, dt="bf16", heads=HQ, T=T, M=ints(1), slot=ints(T), pos=ints(T), theta=1e4,
             rot=torch.zeros((T, (HQ + HK) * DH), dtype=BF), ld_rot=(HQ + HK) * DH, pages=pool())
    a.update(kw)
    S.seer_kv_append(*a.values())


def accept(**kw):
    a = dict(dt="bf16", cached=ints(B), acc=ints(B * 5), n=ints(B), B=B, draft=5, pages=pool(), out=ints(B))
    a.update(kw)
    S.seer_kv_accept(*a.values())


def causal(**kw):
    x = torch.zeros((T, W), dtype=BF)
    a = dict(q=x, ld_q=W, k=x[:, HQ * DH:], ld_k=W, v=x[:, (HQ + HK) * DH:], ld_v=W, o=torch.zeros((T, HQ * DH), dtype=BF), ld_o=HQ * DH,
             dt="bf16", cu=ints(B + 1), B=B, T=T, hq=HQ, hk=HK, dh=DH)
    a.update(kw)
    S.seer_attention_causal(*a.values())


def tree(**kw):
    a = dict(q=torch.zeros((T, HQ * DH), dtype=BF), ld_q=HQ * DH, o=torch.zeros((T, HQ * DH), dtype=BF), ld_o=HQ * DH, dt="bf16", cu=ints(B + 1),
             kv=ints(B), mask=ints(T, torch.int64), B=B, T=T, heads=HQ, draft=4, pages=pool(), ws=torch.zeros(64, dtype=torch.uint8), ws_bytes=64)
    a.update(kw)
    S.seer_attention_tree(*a.values())


CASES = [
    (tables, dict(cached=ints(B - 1)), "cached_len"), (tables, dict(new=ints(0)), "new_len"), (tables, dict(free=ints(3)), "free_pages"),
    (tables, dict(head=ints(0)), "free_head"), (tables, dict(table=ints(B * 4 - 1)), "table"), (tables, dict(max_pages=5), "table"),
    (tables, dict(parent=ints(T - 1)), "parent"), (tables, dict(cu=ints(B)), "cu_new_out"), (tables, dict(kv=ints(1)), "kv_len_out"),
    (tables, dict(slot=ints(T - 1)), "slot_out"), (tables, dict(pos=ints(T - 1)), "position_out"),
    (tables, dict(mask=ints(T - 1, torch.int64)), "mask_out"), (tables, dict(head_out=ints(0)), "free_head_out"),
    (append, dict(qkv=torch.zeros((T, W), dtype=F16)), "qkv"), (append, dict(dt="f32"), "qkv"), (append, dict(T=T + 1), "qkv"),
    (append, dict(qkv=torch.zeros(T * W - 1, dtype=BF)), "qkv"), (append, dict(heads=HQ + 1, ld=W + 64), "qkv"),
    (append, dict(qkv=torch.zeros(T * W + 8, dtype=BF)[16:]), "qkv"),
    (append, dict(rot=torch.zeros((T, (HQ + HK) * DH), dtype=F32)), "rotated"),
    (append, dict(rot=torch.zeros((T - 1, (HQ + HK) * DH), dtype=BF)), "rotated"), (append, dict(slot=ints(T - 1)), "slot"),
    (append, dict(pos=ints(T - 1)), "position"), (append, dict(M=ints(0)), "M_dev"), (append, dict(pages=pool(F16)), "pool"),
    (accept, dict(dt="f32"), "pool"), (accept, dict(cached=ints(1)), "cached_len"), (accept, dict(acc=ints(9)), "accepted"),
    (accept, dict(n=ints(1)), "n_accepted"), (accept, dict(out=ints(1)), "len_out"), (accept, dict(pages=pool(requests=1)), "table"),
    (causal, dict(q=torch.zeros((T, W), dtype=F32)), "q is"), (causal, dict(dt="f16"), "q is"), (causal, dict(T=T + 1), "q:"),
    (causal, dict(k=torch.zeros((T - 1, HK * DH), dtype=BF), ld_k=HK * DH), "k:"), (causal, dict(v=torch.zeros((T, DH), dtype=BF)), "v:"),
    (causal, dict(o=torch.zeros((T - 1, HQ * DH), dtype=BF)), "o:"), (causal, dict(o=torch.zeros((T, HQ * DH), dtype=F32)), "o is"),
    (causal, dict(cu=ints(B)), "cu_seqlens"), (causal, dict(hk=HQ), "v:"),
    (tree, dict(q=torch.zeros((T, HQ * DH), dtype=F32)), "q is"), (tree, dict(T=T + 1), "q:"), (tree, dict(o=torch.zeros(T, dtype=BF)), "o:"),
    (tree, dict(cu=ints(B)), "cu_new"), (tree, dict(kv=ints(1)), "kv_len"), (tree, dict(ws_bytes=65), "ws"), (tree, dict(ws_bytes=-1), "range"),
    (tree, dict(ws=torch.zeros((8, 16), dtype=torch.uint8)[:, :8]), "ws"), (tree, dict(pages=pool(F32)), "pool"),
    (tree, dict(pages=pool(requests=1)), "table")]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_calls_refuse_tensors_that_do_not_hold_what_they_name(i):
    call, kw, name = CASES[i]
    with pytest.raises(ValueError, match=name):
        call(**kw)


@pytest.mark.parametrize("call", [tables, append, accept, causal, tree])
def test_whole_tensors_go_on_to_the_device_check(call):
    """Tensors that hold enough, column blocks and larger buffers among them, are refused for their device alone."""
    if torch.cuda.is_available():
        with pytest.raises(ValueError, match="device"):
            call()
    else:
        with pytest.raises(RuntimeError):                   # no device to compare with
            call()


def test_pools_of_other_types_are_refused():
    with pytest.raises(ValueError):
        S.make_pages(torch.zeros((160, 2 * HK * DH), dtype=torch.uint8), torch.zeros((2, 4), dtype=torch.int32), 10, 16, 4, HK, DH)
