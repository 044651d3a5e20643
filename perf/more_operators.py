"""Cases of a paged K/V cache under a budget: rotary positions of either layout, of part
of a head and scaled for long contexts (rows of heads, and rows appended to the cache),
attention weight accumulated per cached row, the choice of the rows to keep by it, and
their moves.

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
MAX_DRAFT = 64                                  # new rows of a request that look, at most

# scalings: (factor, low, high, original length, magnitude)
SCALES = dict(none=(1.0, 1.0, 1.0, 1, 1.0), linear=(4.0, 1.0, 1.0, 1, 1.0), turns=(8.0, 1.0, 4.0, 8192, 1.0),
              pairs=(16.0, 1.0, 32.0, 4096, 1.25))


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one decode step's queries and keys of a batch of 64, a quarter of each head turned: all latency
        dict(name="rotate_step_b64", op="rotate", dtype="bf16", heads=40, dh=128, rows=64, rd=32, inter=False,
             scaling="none", theta=10000.0, top=8000, pad=0, shape=1),
        # prompts' queries of a model with interleaved pairs, half of each head, stretched context
        dict(name="rotate_prompts", op="rotate", dtype="bf16", heads=32, dh=128, rows=17901, rd=64, inter=True,
             scaling="pairs", theta=10000.0, top=60000, pad=0, shape=2),
        # one decode step's rows of a batch of 64 whose caches have lost rows
        dict(name="append_step_b64", op="append", dtype="bf16", hq=32, hk=8, dh=128, rd=128, inter=True, scaling="turns",
             theta=500000.0, page=16, cached="200~4000x64", new="1x64", gone="0~30000x64", pad=0, spare=0, shape=3),
        # ragged prompts of a long-context model
        dict(name="append_prompts_b16", op="append", dtype="bf16", hq=32, hk=8, dh=128, rd=64, inter=False, scaling="turns",
             theta=500000.0, page=64, cached="0~20000x16", new="300~4000x16", gone="0~60000x16", pad=0, spare=100, shape=4),
        # two interactive requests, one token each
        dict(name="mass_decode_b2", op="mass", dtype="bf16", hq=32, hk=8, dh=128, page=16, cached="700,433", new="1x2",
             gone="0,90", window=1, accept=False, keep=1.0, pad=0, shape=5),
        # a serving batch, one token each over caches of very different lengths
        dict(name="mass_decode_b64", op="mass", dtype="bf16", hq=32, hk=8, dh=128, page=16, cached="200~8000x64",
             new="1x64", gone="0~30000x64", window=1, accept=False, keep=1.0, pad=0, shape=6),
        # prompts just stored, looked at by their last rows
        dict(name="mass_prompts_b16", op="mass", dtype="f16", hq=32, hk=8, dh=128, page=64, cached="0x16",
             new="300~4000x16", gone="0x16", window=64, accept=False, keep=0.0, pad=0, shape=7),
        # a small fp32 model's accepted drafts, earlier weight fading
        dict(name="mass_accepted_f32_b5", op="mass", dtype="f32", hq=4, hk=2, dh=64, page=8, cached="1,17,130,255,900",
             new="24x5", gone="0~50x5", window=24, accept=True, keep=0.9375, pad=0, shape=8),
        # a serving batch back to its budgets
        dict(name="select_b64", op="select", length="200~8000x64", budget=0.5, sinks=4, recent=64, shape=9),
        # one long document cut to an eighth
        dict(name="select_b1", op="select", length="120000", budget=0.125, sinks=4, recent=512, shape=10),
        # a ragged batch of prompts cut to half
        dict(name="evict_b16", op="evict", dtype="bf16", hk=8, dh=128, page=64, length="300~8000x16", budget=0.5, sinks=4,
             recent=64, shape=11),
        # a page's worth of rows from each of a few short caches
        dict(name="evict_b4", op="evict", dtype="bf16", hk=8, dh=128, page=16, length="528x4", budget=0.97, sinks=4,
             recent=32, shape=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "mass", "mass", "select", "evict"])
    shape = rng.randrange(1 << 20)
    page = rng.choice([8, 16, 32, 64, 128, 256])
    hk, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
    dh = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    c = dict(op=op, shape=shape)
    if op in ("rotate", "append"):
        wide = rng.choice([dh, dh, 80 if op == "rotate" else dh])
        c.update(dtype=dtype, dh=wide, rd=rng.choice([wide, wide // 2, wide // 4, 4 * rng.randint(1, wide // 4)]),
                 inter=rng.random() < 0.5, scaling=rng.choice(sorted(SCALES)), theta=rng.choice([10000.0, 500000.0]),
                 pad=rng.choice([0, 0, 64]))
        if op == "rotate":
            heads = hk * rng.choice([1, g])
            c.update(heads=heads, rows=_log_int(rng, 1, max(2, min(40000, 70_000_000 // (heads * wide)))),
                     top=_log_int(rng, 100, 1_000_000))
            return c
        b = _log_int(rng, 1, 64)
        top = max(1, min(4000, 60_000_000 // (hk * (g + 2) * dh * b)))
        c.update(hq=hk * g, hk=hk, page=page, cached=f"{rng.choice([0, 1, 50])}~{_log_int(rng, 60, 20000)}x{b}",
                 new=f"1~{_log_int(rng, 1, top)}x{b}", gone=f"0~{_log_int(rng, 2, 100000)}x{b}",
                 spare=rng.choice([0, 0, 1, 37]))
        return c
    if op == "mass":
        accept = rng.random() < 0.25
        b = _log_int(rng, 1, 64)
        look = rng.choice([1, 1, _log_int(rng, 1, MAX_DRAFT)])
        per_key = hk * dh * (8 if dtype == "f32" else 2) * max(1, look * g // 16)
        top = max(64, min(16000, 200_000_000 // (per_key * b)))
        new = f"1~{max(1, look)}x{b}" if accept or rng.random() < 0.5 else f"1~{_log_int(rng, 1, top)}x{b}"
        c.update(dtype=dtype, hq=hk * g, hk=hk, dh=dh, page=page, new=new, gone=f"0~{_log_int(rng, 2, 5000)}x{b}",
                 cached=f"{rng.choice([0, 1, 60]) if b > 3 else 20}~{_log_int(rng, 64, top)}x{b}", window=look, accept=accept,
                 keep=rng.choice([1.0, 0.0, 0.9375]), pad=rng.choice([0, 0, 64]))
        return c
    b = _log_int(rng, 1, 256 if op == "select" else 32)
    top = _log_int(rng, 1000, max(1001, min(120000, 400_000 // b if op == "select" else 80_000_000 // (hk * dh * b))))
    least = rng.choice([0, 1, 30]) if b > 3 else top // 8
    c.update(length=f"{least}~{top}x{b}", budget=rng.choice([0.125, 0.5, 0.9, 0.99]), sinks=rng.choice([0, 1, 4]),
             recent=rng.choice([r for r in (0, 1, 32, 64, 512) if r <= max(1, top // 128)]))
    if op == "evict":
        c.update(dtype=dtype, hk=hk, dh=dh, page=page)
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
    """Lengths and accepted paths of a case (host lists)."""
    rng = random.Random(case["shape"])
    s = {k: _lengths(case[k], rng) for k in ("cached", "new", "gone", "length") if k in case}
    if case.get("accept"):                       # a path of the draft, at least its first row
        s["accepted"] = [sorted(rng.sample(range(n), rng.randint(1, n))) for n in s["new"]]
    if "length" in s:
        s["budget"] = [int(n * case["budget"]) for n in s["length"]]
        s["gone"] = [rng.choice([0, 0, rng.randrange(1, 40000)]) for _ in s["length"]]
    return s


def _pages_of(rows, page):
    return -(-rows // page)


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _rates(case):
    """Angle per position of each pair, in 64 bits."""
    rd, theta = case["rd"], case["theta"]
    f, lo, hi, length, _ = SCALES[case["scaling"]]
    i = torch.arange(rd // 2, dtype=torch.float64)
    rate = theta ** (-2.0 * i / rd)
    if case["scaling"] == "linear":
        return rate / f
    if case["scaling"] == "turns":
        g = ((length * rate / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1)
        return rate * (g + (1 - g) / f)
    if case["scaling"] == "pairs":
        a = max(math.floor(rd * math.log(length / (2 * math.pi * hi)) / (2 * math.log(theta))), 0)
        b = min(math.ceil(rd * math.log(length / (2 * math.pi * lo)) / (2 * math.log(theta))), rd - 1)
        t = ((i - a) / (b - a if b > a else 0.001)).clamp(0, 1)
        return rate * (1 - t + t / f)
    return rate


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

    def weights(self, rows, cols):
        """Accumulated weights: most rows little, a few much, some none (so that ties occur)."""
        w = torch.randn(rows, cols, device=self.dev, generator=self.gen).mul_(2.0).exp_()
        none = torch.rand(rows, cols, device=self.dev, generator=self.gen) < 0.02
        return w.masked_fill_(none, 0.0)


def _pool(st, case, m, total):
    """A pool of shuffled pages and the requests' table; unused entries are -1."""
    page, B = case["page"], len(total)
    need = [_pages_of(t, page) for t in total]
    st["max_pages"] = max(max(need), 1)
    st["n_pages"] = sum(need) + 7
    order = m.order(st["n_pages"])
    first = torch.tensor([sum(need[:i]) for i in range(B)], device=m.dev)[:, None]
    col = torch.arange(st["max_pages"], device=m.dev)[None, :]
    have = torch.tensor(need, device=m.dev)[:, None]
    st["table"] = torch.where(col < have, order[(first + col).clamp(max=st["n_pages"] - 1)], -1).to(torch.int32)
    st["kv"] = m.normal(st["n_pages"] * page, 2 * case["hk"] * case["dh"], TDT[case["dtype"]])
    if own:
        from paper_2607_14557_gb300 import seer as S
        st["pages"] = S.make_pages(st["kv"], st["table"], st["n_pages"], page, st["max_pages"], case["hk"], case["dh"])


def _births(m, lengths, gone, ld):
    """Positions of cached rows: of the length + gone tokens so far, the last ones in order behind others in any."""
    out = torch.full((len(lengths), ld), -1, dtype=torch.int32, device=m.dev)
    for b, (n, lost) in enumerate(zip(lengths, gone)):
        if lost == 0:
            out[b, :n] = torch.arange(n, device=m.dev)
            continue
        tail = min(n, 600)
        early = m.order(n - tail + lost)[:n - tail]
        out[b, :n - tail] = early
        out[b, n - tail:n] = torch.arange(n - tail + lost, n + lost, device=m.dev)
    return out


def prepare(case, seed):
    sh = _shape(case)
    m = _Maker(case, seed)
    st = dict(case)
    st.update(sh)
    op = case["op"]
    i32 = dict(dtype=torch.int32, device=m.dev)
    if op in ("rotate", "append"):
        st["rate"] = _rates(case).to(m.dev)
        f, lo, hi, length, magnitude = SCALES[case["scaling"]]
        st["magnitude"] = magnitude
        if own:
            from paper_2607_14557_gb300 import seer as S
            st["rotary"] = S.make_rotary(case["theta"], case["rd"], interleaved=case["inter"], scaling=case["scaling"],
                                         factor=f, low=lo, high=hi, original_len=length, magnitude=magnitude)
    if op == "rotate":
        dt, w = TDT[case["dtype"]], case["heads"] * case["dh"]
        st["x"] = m.normal(case["rows"], w + case["pad"], dt)
        st["position"] = torch.randint(case["top"], (case["rows"],), device=m.dev, generator=m.gen).to(torch.int32)
        st["out"] = torch.zeros(case["rows"], w, dtype=dt, device=m.dev)
        return st
    if op in ("select", "evict"):
        B, L = len(sh["length"]), sh["length"]
        st["ld"] = max(max(L), 1)
        st["len_dev"], st["gone_dev"], st["budget_dev"] = m.ints(L), m.ints(sh["gone"]), m.ints(sh["budget"])
        st["mass"], st["birth"] = m.weights(B, st["ld"]), _births(m, L, sh["gone"], st["ld"])
        st["ld_move"] = max([min(n, k - n) for k, n in zip(L, sh["budget"])] + [1])
        st["len_out"], st["gone_out"], st["n_moves"] = (torch.zeros(B, **i32) for _ in range(3))
        st["move_from"], st["move_to"] = (torch.full((B, st["ld_move"]), -1, **i32) for _ in range(2))
        if op == "evict":                        # the moves that the choice has made
            _pool(st, case, m, L)
            _plain_select(st)
        return st
    cached, new = sh["cached"], sh["new"]
    B = len(cached)
    dt = TDT[case["dtype"]]
    width = case["hq"] * case["dh"]
    left = [len(a) for a in sh["accepted"]] if case.get("accept") else new
    total = [c + n for c, n in zip(cached, left)]
    _pool(st, case, m, total)
    T = sum(new)
    st["rows"], st["cap"] = T, T + case.get("spare", 0)
    st["cu"], st["gone_dev"] = m.ints(_starts(new)), m.ints(sh["gone"])
    st["kv_len"] = m.ints(total)
    if op == "append":
        st["qkv"] = m.normal(st["cap"], width + 2 * case["hk"] * case["dh"] + case["pad"], dt)
        rows = torch.repeat_interleave(torch.arange(B, device=m.dev), m.ints(new).long(), output_size=T)
        row = torch.arange(T, device=m.dev) - st["cu"].long()[rows] + m.ints(cached).long()[rows]
        slot = st["table"].long()[rows, row // case["page"]] * case["page"] + row % case["page"]
        fill = torch.full((case["spare"],), -1, device=m.dev)   # the spare rows behind have no slot
        st["request"] = rows
        st["slot"] = torch.cat([slot, fill]).to(torch.int32)
        st["position"] = torch.cat([row, fill.clamp(min=0)]).to(torch.int32)
        st["rotated"] = torch.zeros(st["cap"], (case["hq"] + case["hk"]) * case["dh"], dtype=dt, device=m.dev)
        return st
    st["q"] = m.normal(T, width + case["pad"], dt)
    st["ld"] = max(total)
    st["mass"] = m.weights(B, st["ld"])
    st["mass_out"] = torch.zeros(B, st["ld"], device=m.dev)
    st["birth"] = _births(m, cached, sh["gone"], st["ld"])
    st["accepted_dev"] = st["n_accepted"] = None
    st["draft"] = max(new)
    if case["accept"]:
        st["accepted_dev"] = m.ints([a + [-1] * (st["draft"] - len(a)) for a in sh["accepted"]])
        st["n_accepted"] = m.ints(left)
    st["total"], st["left"], st["kv_cap"] = total, left, sum(total)
    if own:
        from paper_2607_14557_gb300 import seer as S
        st["ws_bytes"] = S.seer_attention_mass_workspace_size(case["dtype"], B, st["kv_cap"], case["hq"], case["hk"],
                                                              case["dh"], case["window"])
        st["ws"] = torch.empty(max(st["ws_bytes"], 16), dtype=torch.uint8, device=m.dev)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return (_OWN if own else _PLAIN)[st["op"]](st)


def _own_rotate(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_rotate(st["x"], st["x"].stride(0), st["dtype"], st["heads"], st["dh"], st["rows"], None, st["position"],
                  st["rotary"], st["out"], st["out"].stride(0))
    return st["out"]


def _own_append(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_kv_append_rotary(st["qkv"], st["qkv"].stride(0), st["dtype"], st["hq"], st["cap"], None, st["slot"],
                            st["position"], st["cu"], st["gone_dev"], len(st["new"]), st["rotary"], st["rotated"],
                            st["rotated"].stride(0), st["pages"])
    return st["rotated"], st["kv"]


def _own_mass(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_attention_mass(st["q"], st["q"].stride(0), st["dtype"], st["cu"], st["kv_len"], st["accepted_dev"],
                          st["n_accepted"], st["draft"], st["window"], len(st["new"]), st["rows"], st["kv_cap"], st["hq"],
                          st["pages"], st["keep"], st["gone_dev"], st["mass"], st["mass_out"], st["birth"], st["ld"],
                          st["ws"], st["ws_bytes"])
    return st["mass_out"], st["birth"]


def _own_select(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_evict_select(st["mass"], st["birth"], st["ld"], st["len_dev"], st["gone_dev"], st["budget_dev"],
                        len(st["length"]), st["sinks"], st["recent"], st["len_out"], st["gone_out"], st["n_moves"],
                        st["move_from"], st["move_to"], st["ld_move"])
    return _select_out(st)


def _own_evict(st):
    from paper_2607_14557_gb300 import seer as S
    S.seer_kv_evict(st["dtype"], st["len_dev"], st["n_moves"], st["move_from"], st["move_to"], st["ld_move"],
                    len(st["length"]), st["pages"], st["mass"], st["birth"], st["ld"])
    return st["kv"], st["mass"], st["birth"]


def _select_out(st):
    return tuple(st[k] for k in ("len_out", "gone_out", "n_moves", "move_from", "move_to"))


def _plain_turn(st, x, position):
    """Heads x [rows, heads, dh] in 32 bits."""
    rd = st["rd"]
    angle = position.double()[:, None] * st["rate"][None, :]
    c, s = (f(angle).float()[:, None] * st["magnitude"] for f in (torch.cos, torch.sin))
    if st["inter"]:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
        return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., rd:]], -1)
    a, b = x[..., :rd // 2], x[..., rd // 2:rd]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., rd:]], -1)


def _plain_rotate(st):
    x = st["x"][:, :st["heads"] * st["dh"]].float().view(-1, st["heads"], st["dh"])
    st["out"].copy_(_plain_turn(st, x, st["position"]).flatten(1))
    return st["out"]


def _plain_append(st):
    hq, hk, dh, T = st["hq"], st["hk"], st["dh"], st["rows"]
    x = st["qkv"][:, :(hq + 2 * hk) * dh].float().view(-1, hq + 2 * hk, dh)
    position = st["position"].clone()
    position[:T] += st["gone_dev"][st["request"]]
    qk = _plain_turn(st, x[:, :hq + hk], position)
    st["rotated"].copy_(qk.flatten(1))
    st["kv"][st["slot"][:T].long()] = torch.cat([qk[:T, hq:], x[:T, hq + hk:]], 1).flatten(1).to(st["kv"].dtype)
    return st["rotated"], st["kv"]


def _looking(st, b):
    """Rows of q that look in request b, and the first one's place among its new rows."""
    n = st["left"][b]
    skip = max(0, n - st["window"])
    cu = _starts(st["new"])[b]
    if st["accepted_dev"] is None:
        return slice(cu + skip, cu + n), skip
    return cu + st["accepted_dev"][b, skip:n].long(), skip


def _keys(st, b, total):
    page = st["page"]
    at = st["table"][b, :_pages_of(total, page)].long()[:, None] * page + torch.arange(page, device=st["kv"].device)
    return st["kv"][at.reshape(-1)[:total], :st["hk"] * st["dh"]]


def _plain_mass(st):
    hq, hk, dh = st["hq"], st["hk"], st["dh"]
    out = st["mass_out"]
    for b, (total, n) in enumerate(zip(st["total"], st["left"])):
        rows, skip = _looking(st, b)
        c = total - n
        q = st["q"][rows, :hq * dh].float().view(n - skip, hk, hq // hk, dh).permute(1, 2, 0, 3)
        k = _keys(st, b, total).float().view(total, hk, dh).permute(1, 2, 0)
        s = torch.matmul(q.reshape(hk, -1, dh), k).view(hk, -1, n - skip, total) / math.sqrt(dh)
        t = torch.arange(total, device=s.device)
        seen = t[None, :] <= c + skip + torch.arange(n - skip, device=s.device)[:, None]
        s = torch.where(seen, s, float("-inf"))
        e = torch.exp(s - s.amax(-1, keepdim=True))
        w = (e / e.sum(-1, keepdim=True)).sum((0, 1, 2))
        w[:c] += st["keep"] * st["mass"][b, :c]
        out[b, :total] = w
        st["birth"][b, c:total] = (t[c:] + st["gone_dev"][b]).int()
    return out, st["birth"]


def _plain_select(st):
    for b, (n, budget) in enumerate(zip(st["length"], st["budget"])):
        k = min(budget, n)
        mass, birth = st["mass"][b, :n], st["birth"][b, :n].long()
        rank = torch.where(birth < st["sinks"], 1, 0)
        rank = torch.where(birth >= n + st["gone_dev"][b].long() - min(st["recent"], k), 2, rank)
        by_mass = torch.sort(mass, descending=True, stable=True).indices
        order = by_mass[torch.sort(rank[by_mass], descending=True, stable=True).indices]
        # within the protected ranks the lower row comes first
        guarded = torch.nonzero(rank == 2).flatten(), torch.nonzero(rank == 1).flatten()
        order = torch.cat([*guarded, order[guarded[0].numel() + guarded[1].numel():]])
        kept = torch.zeros(n, dtype=torch.bool, device=mass.device)
        kept[order[:k]] = True
        moving, holes = torch.nonzero(kept[k:]).flatten() + k, torch.nonzero(~kept[:k]).flatten()
        st["move_from"][b, :moving.numel()] = moving.int()
        st["move_to"][b, :holes.numel()] = holes.int()
        st["n_moves"][b], st["len_out"][b] = moving.numel(), k
    st["gone_out"].copy_(st["gone_dev"] + st["len_dev"] - st["len_out"])
    return _select_out(st)


def _plain_evict(st):
    page, B = st["page"], len(st["length"])
    valid = torch.arange(st["ld_move"], device=st["kv"].device)[None, :] < st["n_moves"][:, None]
    b, i = torch.nonzero(valid, as_tuple=True)
    source, to = st["move_from"].long()[b, i], st["move_to"].long()[b, i]
    table = st["table"].long()

    def rows(t):
        return table[b, t // page] * page + t % page

    st["kv"][rows(to)] = st["kv"][rows(source)]
    for x in (st["mass"], st["birth"]):
        x[b, to] = x[b, source]
    return st["kv"], st["mass"], st["birth"]


_OWN = dict(rotate=_own_rotate, append=_own_append, mass=_own_mass, select=_own_select, evict=_own_evict)
_PLAIN = dict(rotate=_plain_rotate, append=_plain_append, mass=_plain_mass, select=_plain_select, evict=_plain_evict)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    sh = _shape(case)
    op = case["op"]
    if op == "select":
        moves = sum(min(k, n - k) for n, k in zip(sh["length"], sh["budget"]))
        return dict(bytes=8 * sum(sh["length"]) + 24 * len(sh["length"]) + 4 * moves, flops=sum(sh["length"]))
    es = 4 if case["dtype"] == "f32" else 2
    if op == "rotate":
        row = case["heads"] * case["dh"] * es
        return dict(bytes=case["rows"] * (2 * row + 4), flops=case["rows"] * 3 * case["heads"] * case["rd"])
    row = case["hk"] * case["dh"] * es
    if op == "evict":                             # about every second row behind the new end is one of the kept
        moves = sum(k * (n - k) // max(n, 1) for n, k in zip(sh["length"], sh["budget"]))
        return dict(bytes=moves * (4 * row + 24) + 8 * len(sh["length"]), flops=0)
    qrow = case["hq"] * case["dh"] * es
    R = sum(sh["new"])
    if op == "append":
        cap = R + case["spare"]
        return dict(bytes=cap * (2 * qrow + 2 * row + 8) + R * 3 * row,
                    flops=cap * 3 * (case["hq"] + case["hk"]) * case["rd"])
    left = [len(a) for a in sh["accepted"]] if case["accept"] else sh["new"]
    total = [c + n for c, n in zip(sh["cached"], left)]
    look = [min(n, case["window"]) for n in left]
    seen = sum(w * (t - w) + w * (w + 1) // 2 for t, w in zip(total, look))
    return dict(bytes=sum(look) * qrow + sum(total) * (row + 8), flops=2 * case["dh"] * case["hq"] * seen)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return dict(rotate=_exact_rotate, append=_exact_append, mass=_exact_mass, select=_exact_select,
                evict=_exact_evict)[case["op"]](st)


def _exact_turn(st, heads, position):
    """Heads as complex pairs, multiplied by unit numbers of the scaled angles."""
    rd, theta = st["rd"], st["theta"]
    f, lo, hi, length, magnitude = SCALES[st["scaling"]]
    unit = []
    for i in range(rd // 2):
        w = math.exp(-2 * i / rd * math.log(theta))
        if st["scaling"] == "linear":
            w /= f
        elif st["scaling"] == "turns":
            n = length * w / (2 * math.pi)
            w = w if n >= hi else (w / f if n <= lo else w * ((n - lo) + (hi - n) / f) / (hi - lo))
        elif st["scaling"] == "pairs":
            first, last = (math.log(length / n / 2 / math.pi) * rd / 2 / math.log(theta) for n in (hi, lo))
            first, last = max(math.floor(first), 0), min(math.ceil(last), rd - 1)
            t = min(max((i - first) / (last - first if last > first else 0.001), 0.0), 1.0)
            w = w * (1 - t) + w / f * t
        unit.append(w)
    turn = position.double().outer(torch.tensor(unit, dtype=torch.float64, device=heads.device))
    unit = torch.polar(torch.full_like(turn, magnitude), turn)[:, None]
    out = heads.clone()
    part = out[..., :rd]
    if st["inter"]:
        z = torch.view_as_complex(part.unflatten(-1, (rd // 2, 2)).contiguous()) * unit
        part.copy_(torch.view_as_real(z).flatten(-2))
    else:
        z = torch.complex(*part.chunk(2, -1)) * unit
        part.copy_(torch.cat([z.real, z.imag], -1))
    return out


def _exact_rotate(st):
    heads = st["x"][:, :st["heads"] * st["dh"]].double().unflatten(1, (st["heads"], st["dh"]))
    return _exact_turn(st, heads, st["position"]).flatten(1)


def _exact_append(st):
    hq, hk, dh, T = st["hq"], st["hk"], st["dh"], st["rows"]
    heads = st["qkv"][:, :(hq + 2 * hk) * dh].double().unflatten(1, (hq + 2 * hk, dh))
    position = st["position"].tolist()
    cu = _starts(st["new"])
    for b, lost in enumerate(st["gone"]):
        for r in range(cu[b], cu[b + 1]):
            position[r] += lost
    turned = _exact_turn(st, heads[:, :hq + hk], torch.tensor(position, device=heads.device))
    kv = st["kv"].double()
    kv.index_copy_(0, st["slot"][:T].long(), torch.cat([turned[:T, hq:], heads[:T, hq + hk:]], 1).flatten(1))
    return turned.flatten(1), kv


def _exact_mass(st):
    hq, hk, dh = st["hq"], st["hk"], st["dh"]
    out, birth = st["mass_out"].double(), st["birth"].clone()
    first = 0
    for b, n in enumerate(st["left"]):
        c = st["cached"][b]
        pos = torch.arange(c + n, device=out.device)
        pool = st["table"][b].long()[pos // st["page"]] * st["page"] + pos % st["page"]
        k = st["kv"].index_select(0, pool)[:, :hk * dh].double().unflatten(1, (hk, dh))
        which = st["accepted"][b] if st["accept"] else list(range(n))
        which = [(i, r) for i, r in enumerate(which)][-st["window"]:]
        q = st["q"][[first + r for _, r in which]].double()
        hidden = pos[None, :] > torch.tensor([c + i for i, _ in which], device=out.device)[:, None]
        sums = torch.zeros(c + n, dtype=torch.float64, device=out.device)
        for h in range(hq):
            s = q[:, h * dh:(h + 1) * dh] @ k[:, h * hk // hq].T * dh ** -0.5
            sums += torch.softmax(s.masked_fill(hidden, -math.inf), 1).sum(0)
        sums[:c] += st["mass"][b, :c].double() * st["keep"]
        out[b, :c + n] = sums
        birth[b, c:c + n] = pos[c:].int() + st["gone"][b]
        first += st["new"][b]
    return out, birth


def _exact_select(st):
    kept_len, gone, counts = [], [], []
    ld = st["ld_move"]
    moves = [[], []]
    for b, n in enumerate(st["length"]):
        mass, birth = st["mass"][b, :n].tolist(), st["birth"][b, :n].tolist()
        k = min(st["budget"][b], n)
        young = n + st["gone"][b] - min(st["recent"], k)

        def key(t):
            if birth[t] >= young:
                return (0, 0.0, t)
            return (1, 0.0, t) if birth[t] < st["sinks"] else (2, -mass[t], t)

        kept = sorted(sorted(range(n), key=key)[:k])
        inside = set(kept)
        source, to = [t for t in kept if t >= k], [t for t in range(k) if t not in inside]
        for out, rows in zip(moves, (source, to)):
            out.append(rows + [-1] * (ld - len(rows)))
        kept_len.append(k)
        gone.append(st["gone"][b] + n - k)
        counts.append(len(source))
    return tuple(torch.tensor(v, dtype=torch.int32) for v in (kept_len, gone, counts, *moves))


def _exact_evict(st):
    kv, mass, birth = st["kv"].double(), st["mass"].double(), st["birth"].clone()
    table, page = st["table"].tolist(), st["page"]
    counts, source, to = st["n_moves"].tolist(), st["move_from"].tolist(), st["move_to"].tolist()
    for b, count in enumerate(counts):
        if count == 0:
            continue
        pool = [[table[b][t // page] * page + t % page for t in rows[b][:count]] for rows in (source, to)]
        kv[pool[1]] = kv[pool[0]]
        for x in (mass, birth):
            x[b, to[b][:count]] = x[b, source[b][:count]]
    return kv, mass, birth
