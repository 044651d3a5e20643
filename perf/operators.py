"""Cases of the paged K/V cache operators: page tables, appending rotated rows,
causal attention over packed prompts, attention of drafted tokens over the pages,
keeping the accepted drafts.

  own            False: plain torch; True: the framework's entry points
  listed()       the cases
  draw(rng)      one more case of the same ranges
  prepare(c, s)  what a user's program holds before the call
  run(state)     one pass; returns its outputs
  work(c)        bytes and operations that one pass cannot do without
  exact(c, s)    the outputs in 64 bits

A case's lengths follow from its texts ("200~8000x64": 64 lengths, their logarithm
uniform; "5,1,30": those) and its `shape` number, so they are the same for every seed.
"""
import math
import random

import torch

own = False

TDT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_DRAFT = 64                                  # drafted rows of a request


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one decode step of a small batch: the smallest call, all latency
        dict(name="tables_decode_b8", op="tables", cached="100~4000x8", new="1x8", page=16, tree=False, shape=1),
        # prompts of a whole queue admitted at once
        dict(name="tables_prompts_b256", op="tables", cached="0x256", new="16~2000x256", page=64, tree=False, shape=2),
        # one decode step's rows of a batch of 64
        dict(name="append_step_b64", op="append", dtype="bf16", hq=32, hk=8, dh=128, page=16, cached="200~8000x64",
             new="1x64", pad=0, spare=0, theta=10000.0, shape=3),
        # ragged prompts' rows, whole K/V of a layer, far positions
        dict(name="append_prompts_b16", op="append", dtype="bf16", hq=32, hk=8, dh=128, page=64, cached="0~20000x16",
             new="300~4000x16", pad=0, spare=100, theta=500000.0, shape=4),
        # a small fp32 model's prompts, one of a single token
        dict(name="causal_f32_b5", op="causal", dtype="f32", hq=4, hk=2, dh=64, new="1,17,130,255,300", pad=0, spare=0,
             shape=5),
        # a ragged batch of prompts, grouped heads
        dict(name="causal_ragged_b16", op="causal", dtype="bf16", hq=32, hk=8, dh=128, new="32~4000x16", pad=0,
             spare=50, shape=6),
        # one video-length prompt (16 frames of 729 rows and the question)
        dict(name="causal_video_b1", op="causal", dtype="bf16", hq=32, hk=8, dh=128, new="11792", pad=0, spare=0,
             shape=7),
        # two interactive requests, one token each
        dict(name="decode_b2", op="tree", dtype="bf16", hq=32, hk=8, dh=128, page=16, cached="700,433", new="1x2",
             pad=0, spare=0, tree=False, shape=8),
        # a serving batch, one token each over caches of very different lengths
        dict(name="decode_b64", op="tree", dtype="bf16", hq=32, hk=8, dh=128, page=16, cached="200~8000x64", new="1x64",
             pad=0, spare=0, tree=False, shape=9),
        # trees of drafted tokens over long and short caches
        dict(name="tree_b12", op="tree", dtype="f16", hq=32, hk=8, dh=128, page=64, cached="500~12000x12", new="16~64x12",
             pad=0, spare=20, tree=True, shape=10),
        # accepted paths of one request, and of a large batch
        dict(name="accept_b1", op="accept", dtype="bf16", hk=8, dh=128, page=16, cached="1000", draft=24, shape=11),
        dict(name="accept_b128", op="accept", dtype="bf16", hk=8, dh=128, page=64, cached="200~8000x128", draft=64,
             shape=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "append", "causal", "causal", "tree", "tree", "accept"])
    shape = rng.randrange(1 << 20)
    page = rng.choice([8, 16, 32, 64, 128, 256])
    hk, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
    dh = rng.choice([64, 128, 128])
    c = dict(op=op, shape=shape)
    if op == "tables":
        tree = rng.random() < 0.5
        b = _log_int(rng, 1, 512)
        new = f"1~{_log_int(rng, 1, 64)}" if tree else f"1~{_log_int(rng, 1, max(1, min(8000, 400000 // b)))}"
        c.update(cached=f"{rng.choice([0, 1, 50])}~{_log_int(rng, 60, 20000)}x{b}", new=f"{new}x{b}", page=page, tree=tree)
        return c
    c.update(dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if op == "accept":
        b = _log_int(rng, 1, 256)
        c.update(hk=hk, dh=dh, page=page, cached=f"{rng.choice([0, 1, 90])}~{_log_int(rng, 100, 4000)}x{b}",
                 draft=rng.randint(8, MAX_DRAFT))
        return c
    c.update(hq=hk * g, hk=hk, dh=dh, pad=rng.choice([0, 0, 64]), spare=rng.choice([0, 0, 1, 37]))
    rows_kb = hk * (g + 2) * dh                  # values of a packed row
    if op == "append":
        b = _log_int(rng, 1, 64)
        top = max(1, min(4000, 60_000_000 // (rows_kb * b)))
        c.update(page=page, cached=f"{rng.choice([0, 1, 50])}~{_log_int(rng, 60, 20000)}x{b}",
                 new=f"1~{_log_int(rng, 1, top)}x{b}", theta=rng.choice([10000.0, 500000.0, 0.0]))
    elif op == "causal":
        b = _log_int(rng, 1, 16)
        top = int(math.sqrt(11792.0 ** 2 * 4096 / (hk * g * dh) / b / (16 if c["dtype"] == "f32" else 1)))
        c.update(new=f"1~{_log_int(rng, 1, min(top, 11792))}x{b}")
    else:
        b = _log_int(rng, 1, 64)
        tree = rng.random() < 0.6
        top = max(64, min(16000, 200_000_000 // (hk * dh * b)))
        n = _log_int(rng, 1, MAX_DRAFT)
        c.update(page=page, cached=f"{rng.choice([0, 1, 60])}~{_log_int(rng, 64, top)}x{b}", new=f"1~{n}x{b}", tree=tree)
    return c


def _lengths(text, rng):
    head, _, count = text.partition("x")
    count = int(count or 1)
    if "," in head:
        return [int(v) for v in head.split(",")]
    lo, _, hi = head.partition("~")
    lo, hi = int(lo), int(hi or lo)
    lo, hi = min(lo, hi), max(lo, hi)
    if lo == hi:
        return [lo] * count
    return [min(hi, _log_int(rng, max(lo, 1), hi) if rng.random() < 0.95 else lo) for _ in range(count)]


def _shape(case):
    """Lengths, parents and accepted paths of a case (host lists)."""
    rng = random.Random(case["shape"])
    s = {}
    if "cached" in case:
        s["cached"] = _lengths(case["cached"], rng)
    if "new" in case:
        s["new"] = _lengths(case["new"], rng)
    if case.get("tree"):                          # a parent is an earlier row of the draft, or the last cached row
        s["parent"] = [[-1 if i == 0 else rng.randrange(max(-1, i - 9), i) for i in range(n)] for n in s["new"]]
    if case["op"] == "accept":
        s["accepted"] = []
        for _ in s["cached"]:
            n = rng.choice([0, 1, 2, 3, 4, 5])
            s["accepted"].append(sorted(rng.sample(range(n, case["draft"]), min(n, case["draft"] - n))))
    return s


def _pages_of(rows, page):
    return -(-rows // page)


def _masks(parents):
    """Ancestor bits of every row of one draft, as signed 64-bit numbers."""
    bits = []
    for i, p in enumerate(parents):
        bits.append((1 << i) | (bits[p] if p >= 0 else 0))
    return [b - (1 << 64) if b >> 63 else b for b in bits]


# ------------------------------------------------------------------ the states
class _Maker:
    def __init__(self, case, seed):
        self.dev = torch.device("cuda", torch.cuda.current_device())
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(seed * 1000003 + case["shape"])

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.dev)

    def normal(self, rows, cols, dtype):
        out = torch.empty(rows, cols, dtype=dtype, device=self.dev)
        step = max(1, (1 << 27) // cols)
        for r in range(0, rows, step):
            out[r:r + step] = torch.randn(min(step, rows - r), cols, device=self.dev, generator=self.gen)
        return out

    def order(self, n):
        return torch.randperm(n, device=self.dev, generator=self.gen).to(torch.int32)


def prepare(case, seed):
    sh = _shape(case)
    m = _Maker(case, seed)
    st = dict(case)
    st.update(sh)
    op = case["op"]
    dev = m.dev
    if op == "causal":
        dt = TDT[case["dtype"]]
        T, w = sum(sh["new"]), (case["hq"] + 2 * case["hk"]) * case["dh"]
        st["rows"], st["cap"] = T, T + case["spare"]
        st["qkv"] = m.normal(st["cap"], w + case["pad"], dt)
        st["o"] = torch.zeros(st["cap"], case["hq"] * case["dh"], dtype=dt, device=dev)
        st["cu"] = m.ints([sum(sh["new"][:i]) for i in range(len(sh["new"]) + 1)])
        return st
    page, B = case["page"], len(sh["cached"])
    new = sh.get("new", [case.get("draft", 0)] * B)
    total = [c + n for c, n in zip(sh["cached"], new)]
    st["max_pages"] = max(_pages_of(t, page) for t in total)
    need = [_pages_of(t, page) for t in total]
    st["n_pages"] = sum(need) + 7
    order = m.order(st["n_pages"])
    st["cached_dev"] = m.ints(sh["cached"])
    st["new_dev"] = m.ints(new)
    have = [_pages_of(c, page) for c in sh["cached"]] if op == "tables" else need
    # a request's pages, in the order of the shuffled pool; unused entries are -1
    first = torch.tensor([sum(have[:i]) for i in range(B)], device=dev)[:, None]
    col = torch.arange(st["max_pages"], device=dev)[None, :]
    have_t = torch.tensor(have, device=dev)[:, None]
    st["table"] = torch.where(col < have_t, order[(first + col).clamp(max=st["n_pages"] - 1)], -1).to(torch.int32)
    T = sum(new)
    st["rows"], st["cap"] = T, T + case.get("spare", 0)
    i32 = dict(dtype=torch.int32, device=dev)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    if op == "tables":
        st["free"] = order[sum(have):].contiguous()
        st["head"] = m.ints([1])
        st["parent"] = m.ints([p for r in sh["parent"] for p in r]) if case["tree"] else None
        st["cu"], st["kv_len"] = torch.zeros(B + 1, **i32), torch.zeros(B, **i32)
        st["slot"], st["position"] = torch.zeros(T, **i32), torch.zeros(T, **i32)
        st["mask"] = torch.zeros(T, dtype=torch.int64, device=dev) if case["tree"] else None
        st["head_out"] = torch.zeros(1, **i32)
        return st
    dt = TDT[case["dtype"]]
    st["kv"] = m.normal(st["n_pages"] * page, 2 * case["hk"] * case["dh"], dt)
    if op == "accept":
        n = [len(a) for a in sh["accepted"]]
        st["n_accepted"] = m.ints(n)
        st["accepted_dev"] = m.ints([a + [-1] * (case["draft"] - len(a)) for a in sh["accepted"]])
        st["len_out"] = torch.zeros(B, **i32)
    else:
        w = (case["hq"] + 2 * case["hk"]) * case["dh"]
        st["qkv"] = m.normal(st["cap"], w + case["pad"], dt)
        st["cu"] = m.ints(cu)
        st["kv_len"] = m.ints(total)
    if op == "append":
        # rows of requests one after the other; the spare rows behind them have no slot
        rows = torch.repeat_interleave(torch.arange(B, device=dev), st["new_dev"].long(), output_size=T)
        pos = torch.arange(T, device=dev) - st["cu"].long()[rows] + st["cached_dev"].long()[rows]
        slot = st["table"].long()[rows, pos // page] * page + pos % page
        fill = torch.full((case["spare"],), -1, device=dev)
        st["slot"] = torch.cat([slot, fill]).to(torch.int32)
        st["position"] = torch.cat([pos, fill.clamp(min=0)]).to(torch.int32)
        st["rotated"] = torch.zeros(st["cap"], (case["hq"] + case["hk"]) * case["dh"], dtype=dt, device=dev)
    if op == "tree":
        st["o"] = torch.zeros(st["cap"], case["hq"] * case["dh"], dtype=dt, device=dev)
        bits = [b for p in sh["parent"] for b in _masks(p)] if case["tree"] else None
        st["mask"] = torch.tensor(bits, dtype=torch.int64, device=dev) if bits is not None else None
        st["draft"] = max(new)
    if own:
        from paper_2607_14557_gb300 import seer as S
        st["pages"] = S.make_pages(st["kv"], st["table"], st["n_pages"], page, st["max_pages"], case["hk"], case["dh"])
        if op == "tree":
            st["ws_bytes"] = S.seer_attention_tree_workspace_size(case["dtype"], B, case["hq"], case["hk"], case["dh"],
                                                                  st["draft"])
            st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device=dev)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return (_OWN if own else _PLAIN)[st["op"]](st)


def _own_tables(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_page_tables(st["cached_dev"], st["new_dev"], len(st["cached"]), st["page"], st["n_pages"], st["free"],
                       st["free"].numel(), st["head"], st["table"], st["max_pages"], st["rows"], st["parent"], st["cu"],
                       st["kv_len"], st["slot"], st["position"], st["mask"], st["head_out"])
    return _tables_out(st, *(st[k] for k in ("cu", "kv_len", "slot", "position", "mask", "table", "head_out")))


def _own_append(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_kv_append(st["qkv"], st["qkv"].stride(0), st["dtype"], st["hq"], st["cap"], None, st["slot"], st["position"],
                     st["theta"], st["rotated"], st["rotated"].stride(0), st["pages"])
    return st["rotated"], st["kv"]


def _own_causal(st):
    from paper_2607_14557_gb300 import seer as S
    q, k, v = _split(st)
    ld = st["qkv"].stride(0)
    S.seer_attention_causal(q, ld, k, ld, v, ld, st["o"], st["o"].stride(0), st["dtype"], st["cu"], len(st["new"]),
                            st["cap"], st["hq"], st["hk"], st["dh"])
    return st["o"]


def _own_tree(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_attention_tree(st["qkv"], st["qkv"].stride(0), st["o"], st["o"].stride(0), st["dtype"], st["cu"], st["kv_len"],
                          st["mask"], len(st["new"]), st["cap"], st["hq"], st["draft"], st["pages"], st["ws"],
                          st["ws_bytes"])
    return st["o"]


def _own_accept(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_kv_accept(st["dtype"], st["cached_dev"], st["accepted_dev"], st["n_accepted"], len(st["cached"]), st["draft"],
                     st["pages"], st["len_out"])
    return st["kv"], st["len_out"]


def _split(st):
    """q, k and v columns of the packed rows."""
    nq, nk = st["hq"] * st["dh"], st["hk"] * st["dh"]
    x = st["qkv"]
    return x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:nq + 2 * nk]


def _tables_out(st, cu, kv_len, slot, position, mask, table, head):
    out = dict(cu=cu, kv_len=kv_len, slot=slot, position=position, table=table, head=head)
    if mask is not None:
        out["mask"] = mask
    return out


def _plain_tables(st):
    page, B, T = st["page"], len(st["cached"]), st["rows"]
    dev = st["table"].device
    cached, new = st["cached_dev"].long(), st["new_dev"].long()
    total = cached + new
    old, need = (cached + page - 1) // page, (total + page - 1) // page
    taken = need - old
    start = torch.cumsum(taken, 0) - taken + st["head"].long()
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), torch.cumsum(new, 0)])
    col = torch.arange(st["max_pages"], device=dev)[None, :]
    fresh = (col >= old[:, None]) & (col < need[:, None])
    source = (start[:, None] + col - old[:, None]).clamp(0, st["free"].numel() - 1)
    table = torch.where(fresh, st["free"][source], st["table"])
    b = torch.repeat_interleave(torch.arange(B, device=dev), new, output_size=T)
    i = torch.arange(T, device=dev) - cu[b]
    p = cached[b] + i
    slot = table.long()[b, p // page] * page + p % page
    position, mask = p, None
    if st["parent"] is not None:
        up = st["parent"].long()
        node, mask, depth = i, torch.zeros_like(i), torch.full_like(i, -1)
        for _ in range(max(st["new"])):
            alive = node >= 0
            mask = mask | torch.where(alive, torch.ones_like(i) << node.clamp(min=0), 0)
            depth = depth + alive
            node = torch.where(alive, up[cu[b] + node.clamp(min=0)], node)
        position = cached[b] + depth
    return _tables_out(st, cu.int(), total.int(), slot.int(), position.int(), mask, table, (st["head"] + taken.sum()).int())


def _plain_append(st):
    hq, hk, dh = st["hq"], st["hk"], st["dh"]
    x = st["qkv"][:, :(hq + 2 * hk) * dh].float().view(-1, hq + 2 * hk, dh)
    qk, v = x[:, :hq + hk], x[:, hq + hk:]
    if st["theta"] > 0:
        i = torch.arange(dh // 2, dtype=torch.float64, device=x.device)
        angle = st["position"].double()[:, None] * (st["theta"] ** (-2.0 * i / dh))[None, :]
        c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        a, b = qk[..., :dh // 2], qk[..., dh // 2:]
        qk = torch.cat([a * c - b * s, b * c + a * s], -1)
    dt = st["qkv"].dtype
    T = st["rows"]
    st["rotated"].copy_(qk.reshape(qk.shape[0], -1).to(dt))
    st["kv"][st["slot"][:T].long()] = torch.cat([qk[:T, hq:], v[:T]], 1).reshape(T, -1).to(dt)
    return st["rotated"], st["kv"]


def _softmax_rows(s, seen):
    """exp(s - max) / sum over the seen keys; rows that see none are 0."""
    s = torch.where(seen, s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total)


def _plain_causal(st):
    hq, hk, dh = st["hq"], st["hk"], st["dh"]
    q, k, v = _split(st)
    row = 0
    for n in st["new"]:
        qs, ks, vs = (t[row:row + n].float().view(n, -1, dh) for t in (q, k, v))
        j = torch.arange(n, device=q.device)
        seen = (j[None, :] <= j[:, None])[None]
        for h in range(hk):
            g = hq // hk
            s = torch.matmul(qs[:, h * g:(h + 1) * g].transpose(0, 1), ks[:, h].t()) / math.sqrt(dh)
            o = torch.matmul(_softmax_rows(s, seen), vs[:, h])
            st["o"][row:row + n].view(n, hq, dh)[:, h * g:(h + 1) * g] = o.transpose(0, 1).to(st["o"].dtype)
        row += n
    return st["o"]


def _plain_tree(st):
    hq, hk, dh, page = st["hq"], st["hk"], st["dh"], st["page"]
    g = hq // hk
    dev = st["kv"].device
    row = 0
    for b, (c, n) in enumerate(zip(st["cached"], st["new"])):
        total = c + n
        at = (st["table"][b, :_pages_of(total, page)].long()[:, None] * page + torch.arange(page, device=dev)).reshape(-1)
        kv = st["kv"][at[:total]].float().view(total, 2, hk, dh)
        q = st["qkv"][row:row + n, :hq * dh].float().view(n, hk, g, dh).permute(1, 2, 0, 3)
        s = torch.matmul(q, kv[:, 0].permute(1, 2, 0)[:, None]) / math.sqrt(dh)
        j = torch.arange(n, device=dev)
        if st["mask"] is None:
            among = j[None, :] <= j[:, None]
        else:
            among = ((st["mask"][row:row + n, None] >> j[None, :]) & 1) > 0
        seen = torch.cat([torch.ones(n, c, dtype=torch.bool, device=dev), among], 1)
        o = torch.matmul(_softmax_rows(s, seen), kv[:, 1].permute(1, 0, 2)[:, None])
        st["o"][row:row + n] = o.permute(2, 0, 1, 3).reshape(n, hq * dh).to(st["o"].dtype)
        row += n
    return st["o"]


def _plain_accept(st):
    page, w = st["page"], st["draft"]
    B = len(st["cached"])
    c, n = st["cached_dev"].long(), st["n_accepted"].long()
    b = torch.arange(B, device=c.device)
    total = sum(len(a) for a in st["accepted"])
    who = torch.repeat_interleave(b, n, output_size=total)
    k = torch.arange(total, device=c.device) - (torch.cumsum(n, 0) - n)[who]
    table = st["table"].long()

    def rows(p):
        return table[who, p // page] * page + p % page

    st["kv"][rows(c[who] + k)] = st["kv"][rows(c[who] + st["accepted_dev"].long()[who, k])]
    return st["kv"], (c + n).int()


_OWN = dict(tables=_own_tables, append=_own_append, causal=_own_causal, tree=_own_tree, accept=_own_accept)
_PLAIN = dict(tables=_plain_tables, append=_plain_append, causal=_plain_causal, tree=_plain_tree, accept=_plain_accept)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    sh = _shape(case)
    op = case["op"]
    new = sh.get("new", [])
    R = sum(new)
    if op == "tables":
        B, page = len(new), case["page"]
        taken = sum(_pages_of(c + n, page) - _pages_of(c, page) for c, n in zip(sh["cached"], new))
        per_row = 4 + 4 + ((4 + 8) if case["tree"] else 0)
        return dict(bytes=8 * B + 8 * taken + 8 * B + 8 + per_row * R, flops=4 * R)
    es = 4 if case["dtype"] == "f32" else 2
    row = case["hk"] * case["dh"] * es
    if op == "accept":
        moved = sum(len(a) for a in sh["accepted"])
        return dict(bytes=moved * (4 * row + 4) + 12 * len(sh["cached"]), flops=0)
    qrow = case["hq"] * case["dh"] * es
    if op == "append":
        cap = R + case["spare"]
        return dict(bytes=cap * (2 * qrow + 2 * row + 8) + R * 3 * row,
                    flops=cap * 3 * (case["hq"] + case["hk"]) * case["dh"])
    per_pair = 4 * case["dh"] * case["hq"]
    if op == "causal":
        return dict(bytes=R * (2 * qrow + 2 * row), flops=per_pair * sum(n * (n + 1) // 2 for n in new))
    seen = sum(n * c for c, n in zip(sh["cached"], new))
    if case["tree"]:
        seen += sum(bin(b & ((1 << 64) - 1)).count("1") for p in sh["parent"] for b in _masks(p))
    else:
        seen += sum(n * (n + 1) // 2 for n in new)
    return dict(bytes=R * 2 * qrow + 2 * row * sum(c + n for c, n in zip(sh["cached"], new)), flops=per_pair * seen)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return dict(tables=_exact_tables, append=_exact_append, causal=_exact_causal, tree=_exact_tree,
                accept=_exact_accept)[case["op"]](st)


def _exact_tables(st):
    page = st["page"]
    table, free = st["table"].tolist(), st["free"].tolist()
    head = int(st["head"])
    cu, kv_len, slot, position, mask = [0], [], [], [], []
    for b, (c, n) in enumerate(zip(st["cached"], st["new"])):
        while _pages_of(c, page) * page < c + n and table[b][_pages_of(c, page):].count(-1) > 0:
            nxt = table[b].index(-1)
            if nxt * page >= c + n:
                break
            table[b][nxt] = free[head]
            head += 1
        cu.append(cu[-1] + n)
        kv_len.append(c + n)
        depth = []
        up = st["parent"][cu[-2]:cu[-1]].tolist() if st["parent"] is not None else None
        for i in range(n):
            slot.append(table[b][(c + i) // page] * page + (c + i) % page)
            depth.append(i if up is None else (0 if up[i] < 0 else depth[up[i]] + 1))
            position.append(c + depth[i])
        if up is not None:
            mask += _masks(up)
    t = torch.tensor
    return _tables_out(st, t(cu), t(kv_len), t(slot), t(position), t(mask) if st["parent"] is not None else None, t(table),
                       t([head]))


def _exact_append(st):
    hq, hk, dh, T = st["hq"], st["hk"], st["dh"], st["rows"]
    heads = st["qkv"][:, :(hq + 2 * hk) * dh].double().unflatten(1, (hq + 2 * hk, dh))
    pairs = torch.complex(heads[:, :hq + hk, :dh // 2], heads[:, :hq + hk, dh // 2:])
    if st["theta"] > 0:
        rate = torch.exp(torch.arange(0, dh, 2, dtype=torch.float64, device=pairs.device) * (-math.log(st["theta"]) / dh))
        turn = st["position"].double().outer(rate)
        pairs = pairs * torch.polar(torch.ones_like(turn), turn)[:, None]
    turned = torch.cat([pairs.real, pairs.imag], -1)
    kv = st["kv"].double()
    rows = torch.cat([turned[:T, hq:].flatten(1), heads[:T, hq + hk:].flatten(1)], 1)
    kv.index_copy_(0, st["slot"][:T].long(), rows)
    return turned.flatten(1), kv


def _exact_causal(st):
    hq, hk, dh = st["hq"], st["hk"], st["dh"]
    out = st["o"].double()
    q, k, v = (t.double().unflatten(1, (-1, dh)).transpose(0, 1) for t in _split(st))
    row = 0
    for n in st["new"]:
        for h in range(hq):
            kk, vv = k[h * hk // hq, row:row + n], v[h * hk // hq, row:row + n]
            for i in range(0, n, 2048):
                e = min(n, i + 2048)
                s = q[h, row + i:row + e].mul(dh ** -0.5) @ kk[:e].T
                s.masked_fill_(torch.ones_like(s, dtype=torch.bool).triu(i + 1), -math.inf)
                out[row + i:row + e, h * dh:(h + 1) * dh] = torch.softmax(s, 1) @ vv[:e]
        row += n
    return out


def _exact_tree(st):
    hq, hk, dh, page = st["hq"], st["hk"], st["dh"], st["page"]
    out = st["o"].double()
    cu = 0
    for b, (c, n) in enumerate(zip(st["cached"], st["new"])):
        pos = torch.arange(c + n, device=out.device)
        kv = st["kv"].index_select(0, st["table"][b].long()[pos // page] * page + pos % page).double()
        kv = kv.unflatten(1, (2, hk, dh))
        bits = _masks(st["parent"][b]) if st["mask"] is not None else [(1 << (i + 1)) - 1 for i in range(n)]
        hidden = torch.tensor([[(w >> j) & 1 == 0 for j in range(n)] for w in bits], device=out.device)
        hidden = torch.nn.functional.pad(hidden, (c, 0), value=False)
        for h in range(hq):
            k, v = kv[:, 0, h * hk // hq], kv[:, 1, h * hk // hq]
            s = st["qkv"][cu:cu + n, h * dh:(h + 1) * dh].double() @ k.T * dh ** -0.5
            out[cu:cu + n, h * dh:(h + 1) * dh] = torch.softmax(s.masked_fill(hidden, -math.inf), 1) @ v
        cu += n
    return out


def _exact_accept(st):
    kv = st["kv"].double()
    table, page = st["table"].tolist(), st["page"]
    length = []
    for b, (c, kept) in enumerate(zip(st["cached"], st["accepted"])):
        at = [table[b][(c + j) // page] * page + (c + j) % page for j in range(st["draft"])]
        for k, a in enumerate(kept):
            kv[at[k]] = kv[at[a]]
        length.append(c + len(kept))
    return kv, torch.tensor(length)
