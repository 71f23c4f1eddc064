"""Timing cases of the paged caches: storing rows in pages, attention of one new token over them, and eviction by accumulated mass.

A case is one pass of one operation:

  store   rows of a prompt (merged or not) into the pages of their sequences (`ec_paged_store`)
  decode  one generated token through `layers` layers (`ec_paged_decode_step`)
  freq    one generated token through `layers` layers under the frequency policy: attention that adds to the rows' masses, and the row of
          least mass removed from every sequence (`ec_paged_decode_score_step`, `ec_paged_evict_min`)
  shrink  sequences cut down to a smaller budget by the scores of their last pass: these are stored as the rows' masses, and all but the
          `keep` heaviest rows go (`ec_paged_store` without rows, `ec_paged_evict_min`)

Slot s of sequence b is row s % page of page `page_table[b][s // page]`; pages of a sequence lie anywhere in the pool, as after some time
of serving. `own` chooses between the plain form in torch operations and the library.
"""
from __future__ import annotations

import math

import torch

own = False

RECENT = 25  # newest positions that are never evicted
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest call: a first short exchange in fp32, all of it latency
        dict(name="decode_tiny_f32", op="decode", dtype="f32", B=1, H=4, Hkv=4, D=64, page=16, rows=100, layers=1, ragged=False),
        # a single user's compressed image prompt, as many key/value heads as query heads
        dict(name="decode_b1", op="decode", dtype="bf16", B=1, H=32, Hkv=32, D=128, page=16, rows=641, layers=4, ragged=False),
        # an ordinary serving batch of the long prompts' compressed caches
        dict(name="decode_b16", op="decode", dtype="bf16", B=16, H=32, Hkv=32, D=128, page=32, rows=870, layers=4, ragged=False),
        # a large serving batch with grouped queries, lengths mixed, one place free and one sequence at its first token
        dict(name="decode_b48_ragged", op="decode", dtype="bf16", B=48, H=32, Hkv=4, D=128, page=16, rows=2900, layers=2, ragged=True),
        # one very long cache, uncompressed, five queries to a key head: the largest attention there is
        dict(name="decode_b1_long", op="decode", dtype="bf16", B=1, H=40, Hkv=8, D=128, page=64, rows=131071, layers=2, ragged=False),
        # a token of a single user under the frequency policy, layer-wise
        dict(name="freq_b1", op="freq", dtype="bf16", B=1, H=32, Hkv=32, D=128, page=16, rows=513, layers=4, heads=False, ragged=False),
        # the same for a batch with grouped queries whose heads keep rows of their own
        dict(name="freq_b8_heads", op="freq", dtype="bf16", B=8, H=32, Hkv=8, D=128, page=16, rows=1500, layers=4, heads=True, ragged=True),
        # checking in full precision
        dict(name="freq_f32", op="freq", dtype="f32", B=2, H=8, Hkv=2, D=64, page=8, rows=300, layers=2, heads=False, ragged=False),
        # long prompts cut to a tenth when memory runs short: the largest call of eviction
        dict(name="shrink_b16", op="shrink", dtype="bf16", B=16, Hkv=32, D=128, page=64, rows=8192, keep=820, heads=False, ragged=False),
        # a few sequences cut to a third, head by head
        dict(name="shrink_b3_heads", op="shrink", dtype="f32", B=3, Hkv=8, D=64, page=8, rows=3001, keep=1000, heads=True, ragged=True),
        # one image prompt's merged rows, at the end of a shared prefix that ends inside a page
        dict(name="store_b1", op="store", dtype="bf16", B=1, Hkv=8, D=128, page=16, rows=577, start=37, heads=False, ragged=False),
        # prompts of a whole batch, different lengths
        dict(name="store_b16", op="store", dtype="bf16", B=16, Hkv=32, D=128, page=32, rows=2048, start=0, heads=False, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "decode", "freq", "freq", "shrink", "store"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), D=rng.choice([128, 128, 64]), page=rng.choice([8, 16, 32, 64, 128, 256]))
    c["Hkv"] = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    row = c["Hkv"] * c["D"] * 2 * (4 if c["dtype"] == "f32" else 2)  # bytes of K and V of one position
    if op in ("decode", "freq"):
        c["H"] = c["Hkv"] * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 7, 8, 16) if c["Hkv"] * g <= 64])
        c["layers"] = rng.randint(1, 4)
        most = (800 << 20) // (row * c["layers"])
        c["rows"] = _log(rng, 1 if op == "decode" else 40, min(100000 if op == "decode" else 8000, most))
        c["B"] = _log(rng, 1, max(1, min(64, most // c["rows"])))
        if op == "freq":
            c["heads"] = rng.random() < 0.3
    else:
        most = ((1 << 30) if op == "shrink" else (500 << 20)) // row
        c["rows"] = _log(rng, 64 if op == "shrink" else 1, min(12000, most))
        c["B"] = _log(rng, 1, max(1, min(32, most // c["rows"])))
        c["heads"] = rng.random() < 0.3
        if op == "shrink":
            c["keep"] = max(1, int(c["rows"] * rng.uniform(0.05, 0.9)))
        else:
            c["start"] = rng.randint(0, 100)
    c["ragged"] = c["B"] > 1 and rng.random() < 0.5
    return c


# ------------------------------------------------------------------ inputs
def _groups(case):
    return case["Hkv"] if case.get("heads") else 1


def _rows_of(case):
    """Rows of every sequence before the pass: all the same, or between half and all, and then in a decoding batch of four and more one place
    without a sequence (-1) and one sequence without rows. (They belong to the case, so that the outputs' shapes do.)"""
    n, B = case["rows"], case["B"]
    if not case["ragged"]:
        return [n] * B
    g = torch.Generator()
    g.manual_seed(1000 * n + B)
    got = [int(x) for x in torch.randint(max(1, n // 2), n + 1, (B,), generator=g)]
    got[0] = n
    if case["op"] == "decode" and B >= 4:
        got[B // 2], got[B - 1] = -1, 0
    return got


def _layout(case):
    """Rows before the pass, and slots that every sequence needs."""
    rows = _rows_of(case)
    return rows, [max(r + (1 if case["op"] in ("decode", "freq") else case.get("start", 0)), 0) for r in rows]


def prepare(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    B, Hkv, D, page, G = case["B"], case["Hkv"], case["D"], case["page"], _groups(case)
    L = case.get("layers", 1)
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=gen, device=dev, dtype=torch.float32)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    rows, slots = _layout(case)
    used = [-(-n // page) for n in slots]
    N, most = sum(used) + 3, max(used) + 1
    # pages in any order; -1 where a sequence has none
    order, table = torch.randperm(N, generator=gen, device=dev).to(torch.int32), torch.full((B, most), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    s = dict(case=case, table=table, rows=ints(rows))
    s["k"], s["v"] = (torch.empty((L, N, Hkv, page, D), dtype=dt, device=dev) for _ in range(2))
    for i in range(L):
        # a twentieth of the keys draw much attention, the others little, as in prompts
        gain = torch.where(torch.rand((N, 1, page, 1), generator=gen, device=dev) < 0.05, 4.0, 0.7)
        s["k"][i] = randn(N, Hkv, page, D) * gain
        s["v"][i] = randn(N, Hkv, page, D)
    # positions of a sequence's rows: a merged prompt's anchors, every third position or so
    s["pos"], s["mass"] = torch.zeros((L, N, G, page), dtype=torch.int32, device=dev), torch.zeros((L, N, G, page), device=dev)
    top = max(max(slots), 1)
    if case["op"] in ("decode", "freq"):
        pos = (torch.rand((L, B, G, top), generator=gen, device=dev) < 0.5).to(torch.int32).cumsum(-1, dtype=torch.int32) + torch.arange(top, device=dev, dtype=torch.int32)
        # masses of some hundred tokens: a twentieth apart, in any order, so that which one is the least does not hang on a rounding
        mass = torch.rand((L, B, G, top), generator=gen, device=dev).argsort(-1).float() * 0.05
        j = torch.arange(top, device=dev)
        held = j < s["rows"][:, None]
        b, j = held.nonzero(as_tuple=True)
        p, o = table[b, j // page].long(), j % page
        s["pos"][:, p, :, o] = pos[:, b, :, j]
        s["mass"][:, p, :, o] = mass[:, b, :, j]
        s["q"] = randn(L, B, case["H"], D).to(dt)
        s["kn"], s["vn"] = randn(L, B, Hkv, D).to(dt), randn(L, B, Hkv, D).to(dt)
        s["new_pos"] = ints([2 * top + 5] * B)
        s["out"] = torch.empty_like(s["q"])
    if case["op"] == "freq":
        s["len"], s["keep"], s["seen"] = s["rows"] + 1, s["rows"].clone(), s["new_pos"] + 1
        s["evict"] = 1
    elif case["op"] == "shrink":
        # column sums of a chunk's attention: many light rows, some of them at exactly 0, a few heavy ones
        score = torch.rand((B, G, top), generator=gen, device=dev).pow(-0.7)
        s["src_mass"] = torch.where(torch.rand((B, G, top), generator=gen, device=dev) < 0.03, torch.zeros((), device=dev), score)
        s["src_pos"] = torch.arange(top, device=dev, dtype=torch.int32).expand(B, G, top).contiguous()
        s["len"], s["keep"], s["seen"] = s["rows"], torch.full_like(s["rows"], case["keep"]), s["rows"]
        s["evict"] = max(max(rows) - case["keep"], 1)
    elif case["op"] == "store":
        top = case["rows"]
        s["src_k"], s["src_v"] = randn(B, Hkv, top, D).to(dt), randn(B, Hkv, top, D).to(dt)
        s["src_pos"] = torch.arange(top, device=dev, dtype=torch.int32).expand(B, G, top).contiguous()
        s["src_mass"] = torch.rand((B, G, top), generator=gen, device=dev)
        s["start"] = torch.full_like(s["rows"], case["start"])
    if own:
        from paper_2407_18121_amd import binding as ec
        if case["op"] in ("decode", "freq"):
            fn = ec.EC_FN_PAGED_DECODE_STEP if case["op"] == "decode" else ec.EC_FN_PAGED_DECODE_SCORE_STEP
            s["ws"] = ec.new_workspace(fn, B, case["H"], most * page, D, ec.dtype_code(s["q"]))
        if case["op"] in ("freq", "shrink"):
            s["ws_evict"] = ec.new_workspace(ec.EC_FN_PAGED_EVICT_MIN, B, G, s["evict"], D, ec.dtype_code(s["k"]))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if op == "store":
        (_own_store if own else _plain_store)(s, s["src_k"], s["src_v"], s["start"], s["rows"])
        return {"k": s["k"], "v": s["v"], "pos": s["pos"], "mass": s["mass"]}
    if op == "shrink":
        (_own_store if own else _plain_store)(s, None, None, None, s["rows"])
        (_own_evict if own else _plain_evict)(s, 0)
        return {"k": s["k"], "v": s["v"], "pos": s["pos"], "mass": s["mass"]}
    for i in range(s["case"]["layers"]):
        (_own_decode if own else _plain_decode)(s, i)
        if op == "freq":
            (_own_evict if own else _plain_evict)(s, i)
    return {"out": s["out"], "k": s["k"], "v": s["v"], "pos": s["pos"], **({"mass": s["mass"]} if op == "freq" else {})}


def _own_store(s, k, v, start, rows):
    from paper_2407_18121_amd import binding as ec
    ec.ec_paged_store(k, v, s["src_pos"], s["src_mass"], s["table"], s["k"][0] if k is not None else None, s["v"][0] if k is not None else None,
                      s["pos"][0], s["mass"][0], start, rows)


def _own_decode(s, i):
    from paper_2407_18121_amd import binding as ec
    scale = s["case"]["D"] ** -0.5
    if s["case"]["op"] == "freq":
        ec.ec_paged_decode_score_step(s["q"][i], s["kn"][i], s["vn"][i], s["k"][i], s["v"][i], s["pos"][i], s["mass"][i], s["table"], s["rows"],
                                      s["new_pos"], scale, s["out"][i], s["ws"])
    else:
        ec.ec_paged_decode_step(s["q"][i], s["kn"][i], s["vn"][i], s["k"][i], s["v"][i], s["pos"][i], s["table"], s["rows"], s["new_pos"], scale,
                                s["out"][i], s["ws"])


def _own_evict(s, i):
    from paper_2407_18121_amd import binding as ec
    ec.ec_paged_evict_min(s["k"][i], s["v"][i], s["pos"][i], s["mass"][i], s["table"], s["len"], s["keep"], s["seen"], s["evict"], 1, RECENT,
                          s["ws_evict"])


# ------------------------------------------------------------------ the plain form
def _plain_store(s, k, v, start, rows):
    page = s["case"]["page"]
    top = s["src_pos"].shape[2]
    b, j = (torch.arange(top, device=rows.device) < rows[:, None]).nonzero(as_tuple=True)
    at = j + start[b] if start is not None else j
    p, o = s["table"][b, at // page].long(), at % page
    if k is not None:
        s["k"][0][p, :, o] = k[b, :, j]
        s["v"][0][p, :, o] = v[b, :, j]
    s["pos"][0][p, :, o] = s["src_pos"][b, :, j]
    s["mass"][0][p, :, o] = s["src_mass"][b, :, j]


def _plain_decode(s, i):
    case, table, rows = s["case"], s["table"], s["rows"]
    B, H, Hkv, D, page = case["B"], case["H"], case["Hkv"], case["D"], case["page"]
    k, v, pos, mass = s["k"][i], s["v"][i], s["pos"][i], s["mass"][i]
    live = (rows >= 0).nonzero()[:, 0]
    p, o = table[live, rows[live] // page].long(), (rows[live] % page).long()
    k[p, :, o], v[p, :, o] = s["kn"][i][live], s["vn"][i][live]
    pos[p, :, o] = s["new_pos"][live][:, None].expand(-1, pos.shape[1])
    slots = table.shape[1] * page
    ids = table.long().clamp(min=0)
    dense = lambda x: x[ids].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, slots, D)  # noqa: E731
    seen = torch.arange(slots, device=rows.device) <= rows[:, None]
    x = torch.matmul(s["q"][i].float().view(B, Hkv, H // Hkv, D), dense(k).transpose(2, 3)) * D ** -0.5
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    prob = e / torch.where(total == 0, torch.ones_like(total), total)
    # rows behind a sequence's last hold whatever was there before; their weight is 0
    s["out"][i] = torch.matmul(prob, dense(v).masked_fill(~seen[:, None, :, None], 0.0)).view(B, H, D)
    if case["op"] == "freq":
        add = prob.mean(2) if case["heads"] else prob.mean((1, 2))[:, None]
        b, j = seen.nonzero(as_tuple=True)
        p, o = ids[b, j // page], j % page
        held = torch.where((j < rows[b])[:, None], mass[p, :, o], torch.zeros((), device=rows.device))
        mass[p, :, o] = held + add[b, :, j]


def _plain_evict(s, i):
    case, table, length = s["case"], s["table"], s["len"].long()
    page, heads = case["page"], case["heads"]
    k, v, pos, mass = s["k"][i], s["v"][i], s["pos"][i], s["mass"][i]
    slots = table.shape[1] * page
    ids = table.long().clamp(min=0)
    dense = lambda x: x[ids].permute(0, 2, 1, 3).reshape(table.shape[0], x.shape[1], slots)  # noqa: E731
    at = torch.arange(slots, device=length.device)
    held = (at < length[:, None])[:, None]
    where = dense(pos)
    kept = (where < 1) | (where >= (s["seen"].long() - RECENT)[:, None, None])
    order = torch.where(kept, torch.full((), math.inf, device=length.device), dense(mass)).masked_fill(~held, math.inf)
    order = order.argsort(stable=True)  # the lower slot first among equals; rows that do not exist come last
    gone = (length - s["keep"]).clamp(min=0, max=s["evict"])
    victim = torch.zeros(order.shape, dtype=torch.bool, device=length.device).scatter_(-1, order, (at < gone[:, None])[:, None].expand_as(order))
    left = (length - gone)[:, None, None]
    hb, hg, hs = (victim & (at < left)).nonzero(as_tuple=True)
    mb, mg, ms = (~victim & held & (at >= left)).nonzero(as_tuple=True)
    hp, ho, mp, mo = ids[hb, hs // page], hs % page, ids[mb, ms // page], ms % page
    if heads:
        k[hp, hg, ho], v[hp, hg, ho] = k[mp, mg, mo], v[mp, mg, mo]
    else:
        k[hp, :, ho], v[hp, :, ho] = k[mp, :, mo], v[mp, :, mo]
    pos[hp, hg, ho], mass[hp, hg, ho] = pos[mp, mg, mo], mass[mp, mg, mo]


# ------------------------------------------------------------------ what it costs, and what it is
def work(case):
    rows, _ = _layout(case)
    e, D, Hkv, G, B = 4 if case["dtype"] == "f32" else 2, case["D"], case["Hkv"], _groups(case), case["B"]
    pair = 2 * Hkv * D * e  # K and V of one position
    n = sum(max(r, 0) for r in rows)
    if case["op"] == "store":
        return {"bytes": 2 * n * (pair + 8 * G), "flops": 0}
    if case["op"] == "shrink":
        gone = [max(r - case["keep"], 0) for r in rows]
        moved = sum((r - g) * g / r for r, g in zip(rows, gone))  # survivors of the part that is given up: scores do not go by the slot
        return {"bytes": 2 * n * 8 * G + n * 8 * G + 2 * moved * (pair + 8 * G), "flops": 0}
    live = sum(r >= 0 for r in rows)
    one = {"bytes": n * pair + live * (2 * pair + 2 * case["H"] * D * e + 4 * G) + 4 * B * max(-(-(r + 1) // case["page"]) for r in rows),
           "flops": 4 * case["H"] * D * (n + live)}
    if case["op"] == "freq":
        one["bytes"] += (n + live) * 16 * G + 2 * live * (pair + 8 * G)  # masses read, written and looked through with the positions; one row moved
    return {w: x * case["layers"] for w, x in one.items()}


def exact(case, seed):
    s = prepare(case, seed)
    page, G, heads = case["page"], _groups(case), case.get("heads", False)
    table, rows = s["table"].tolist(), s["rows"].tolist()
    k, v, pos, mass = s["k"], s["v"], s["pos"], s["mass"]

    def places(b, n, first=0):
        at = torch.arange(first, first + n)
        return torch.tensor([table[b][int(x) // page] for x in at], dtype=torch.long), at % page

    if case["op"] in ("store", "shrink"):
        for b, n in enumerate(rows):
            p, o = places(b, n, case.get("start", 0))
            if case["op"] == "store":
                k[0, p, :, o], v[0, p, :, o] = s["src_k"][b, :, :n].transpose(0, 1), s["src_v"][b, :, :n].transpose(0, 1)
            pos[0, p, :, o], mass[0, p, :, o] = s["src_pos"][b, :, :n].T, s["src_mass"][b, :, :n].T
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") if "q" in s else None
    wide = mass.double()
    for i in range(case["layers"] if out is not None else 0):
        for b, n in enumerate(rows):
            if n < 0:
                continue
            p, o = places(b, n + 1)
            k[i, p[n], :, o[n]], v[i, p[n], :, o[n]], pos[i, p[n], :, o[n]] = s["kn"][i, b], s["vn"][i, b], s["new_pos"][b]
            group = case["H"] // case["Hkv"]
            total = torch.zeros((G, n + 1), dtype=torch.float64, device="cuda")
            for h in range(case["H"]):
                x = (k[i, p, h // group, o].double() * s["q"][i, b, h].double()).sum(-1) / math.sqrt(case["D"])
                w = torch.softmax(x, 0)
                out[i, b, h] = (w[:, None] * v[i, p, h // group, o].double()).sum(0)
                total[h // group if heads else 0] += w / (group if heads else case["H"])
            if case["op"] == "freq":
                wide[i, p[n], :, o[n]] = 0.0
                wide[i, p, :, o] += total.T
    if case["op"] in ("freq", "shrink"):
        for i in range(case.get("layers", 1)):
            for b in range(case["B"]):
                n = int(s["len"][b])
                gone = min(max(n - int(s["keep"][b]), 0), s["evict"])
                p, o = places(b, n)
                for g in range(G):
                    at, m = pos[i, p, g, o].tolist(), wide[i, p, g, o].tolist()
                    safe = int(s["seen"][b]) - RECENT
                    weakest = sorted(range(n), key=lambda j: (at[j] < 1 or at[j] >= safe, m[j] if 1 <= at[j] < safe else 0.0, j))[:gone]
                    away = set(weakest)
                    holes = torch.tensor([j for j in range(n - gone) if j in away], dtype=torch.long)
                    movers = torch.tensor([j for j in range(n - gone, n) if j not in away], dtype=torch.long)
                    for x in (pos, wide):
                        x[i, p[holes], g, o[holes]] = x[i, p[movers], g, o[movers]]
                    for x in (k, v):
                        if heads:
                            x[i, p[holes], g, o[holes]] = x[i, p[movers], g, o[movers]]
                        else:
                            x[i, p[holes], :, o[holes]] = x[i, p[movers], :, o[movers]]
    got = {"k": k.double(), "v": v.double(), "pos": pos}
    if out is not None:
        got["out"] = out
    if case["op"] != "decode":
        got["mass"] = wide
    return got
