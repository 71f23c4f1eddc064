"""Timing cases of what brings several new tokens of a sequence into paged caches: pages and slots for them, their queries and keys turned by their
positions and stored, and their attention over all that is cached.

A case is one pass of one operation:

  plan    pages given back and taken for every sequence of a batch, the first slot of its new rows, and for every new token its row in the
          pools and its position (`ec_paged_plan`). Two states of the batch take turns, so that pages come and go in every pass
  rotary  queries and keys of new tokens turned by their positions, keys and values into the pages (`ec_paged_rotary_store`)
  chunk   attention of the new tokens, packed one after the other, over the rows of their sequences up to their own (`ec_paged_chunk_step`)

Slot s of sequence b is row s % page of page `table[b][s // page]`; pages of a sequence lie anywhere in the pool, as after some time of
serving. `own` chooses between the plain form in torch operations and the library.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # every sequence of an ordinary batch gets its next token: one in sixteen needs a page
        dict(name="plan_b16", op="plan", B=16, page=16, rows=870, new=1, kind="same", tight=False),
        # a large batch: prompts arrive in chunks beside generation, sequences end and shrink, and the pool does not hold all that is asked for
        dict(name="plan_b256_mixed", op="plan", B=256, page=32, rows=2900, new=512, kind="mixed", tight=True),
        # one token of each of 16 sequences, as many key/value heads as query heads: all of it latency
        dict(name="rotary_t16", op="rotary", dtype="bf16", T=16, H=32, Hkv=32, D=128, rot=128, interleaved=False, page=16, factor=1.0, last=4096, pad=0),
        # long prompts with grouped queries, positions stretched for a long context
        dict(name="rotary_t8192", op="rotary", dtype="bf16", T=8192, H=32, Hkv=8, D=128, rot=128, interleaved=False, page=64, factor=8.0, last=131072, pad=37),
        # checking in full precision: part of the head, neighbouring elements in pairs, sizes that fill no vector
        dict(name="rotary_t777_f32", op="rotary", dtype="f32", T=777, H=8, Hkv=2, D=64, rot=22, interleaved=True, page=8, factor=1.0, last=8192, pad=5),
        # the smallest call: a short question after a short exchange, in fp32
        dict(name="chunk_tiny_f32", op="chunk", dtype="f32", B=1, H=4, Hkv=4, D=64, page=16, rows=100, new=5, kind="same", lse=False),
        # a user's next turn over a compressed cache
        dict(name="chunk_turn2", op="chunk", dtype="bf16", B=1, H=32, Hkv=32, D=128, page=16, rows=768, new=512, kind="same", lse=False),
        # drafted tokens of a batch looked at in one pass, grouped queries, one place free and one sequence without rows
        dict(name="chunk_b8_draft", op="chunk", dtype="bf16", B=8, H=32, Hkv=8, D=128, page=16, rows=2900, new=5, kind="ragged", lse=False),
        # a serving batch in which an eighth of the sequences bring a chunk of a prompt and the others one token
        dict(name="chunk_b32_mixed", op="chunk", dtype="bf16", B=32, H=32, Hkv=8, D=128, page=32, rows=1500, new=1000, kind="mixed", lse=False),
        # first turns of a batch: nothing is cached yet
        dict(name="chunk_first_b4", op="chunk", dtype="bf16", B=4, H=32, Hkv=32, D=128, page=64, rows=0, new=2048, kind="ragged", lse=True),
        # a chunk of a very long prompt, five queries to a key head: the largest call
        dict(name="chunk_long", op="chunk", dtype="bf16", B=1, H=40, Hkv=8, D=128, page=64, rows=65000, new=2048, kind="same", lse=False),
        # checking in full precision
        dict(name="chunk_b2_f32", op="chunk", dtype="f32", B=2, H=8, Hkv=2, D=128, page=8, rows=577, new=300, kind="ragged", lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rotary", "rotary", "chunk", "chunk", "chunk", "chunk"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if op == "plan":
        B = _log(rng, 1, 256)
        c = dict(op=op, B=B, page=page, rows=_log(rng, 16, 4000), kind=rng.choice(["same", "ragged", "mixed"]), tight=rng.random() < 0.3)
        c["new"] = _log(rng, 1, 512 if c["kind"] == "mixed" else max(1, min(512, 16384 // B)))
        return c
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), D=rng.choice([128, 128, 64]), page=page, Hkv=rng.choice([1, 2, 4, 8, 8, 16, 32, 40]))
    c["H"] = c["Hkv"] * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 7, 8, 16) if c["Hkv"] * g <= 64])
    e = 4 if c["dtype"] == "f32" else 2
    if op == "rotary":
        most = 8192 * 48 * 128 * 2 // ((c["H"] + 2 * c["Hkv"]) * c["D"] * e)
        c.update(T=_log(rng, 1, min(most, 30000)), rot=rng.choice([c["D"], c["D"], c["D"] // 2, 2 * rng.randint(1, c["D"] // 2)]), interleaved=rng.random() < 0.4,
                 factor=rng.choice([1.0, 1.0, 4.0, 16.0]), last=_log(rng, 100, 1000000), pad=rng.choice([0, 0, 1, 40]))
        c["pad"] = min(c["pad"], c["T"] - 1)
        return c
    work = 2048 * (65000 + 1024) * 40 * 128 // (1 if c["dtype"] == "bf16" else 40)  # a product in fp32 takes that much longer
    pair = c["Hkv"] * c["D"] * 2 * e
    c["kind"] = rng.choice(["same", "ragged", "mixed"])
    c["B"] = _log(rng, 1, 48)
    c["new"] = _log(rng, 1, 4096 // (c["B"] if c["kind"] != "mixed" else max(1, c["B"] // 8)))
    tokens = c["new"] * c["B"] if c["kind"] != "mixed" else c["new"] * -(-c["B"] // 8) + c["B"]
    most = min((800 << 20) // (pair * c["B"]), work // (tokens * c["H"] * c["D"]) - c["new"], 65000)
    c["rows"] = rng.choice([0, 1]) if most < 2 or rng.random() < 0.1 else _log(rng, 1, most)
    c["lse"] = rng.random() < 0.3
    return c


# ------------------------------------------------------------------ inputs
def _layout(case):
    """Rows before the pass and new tokens of every sequence. They belong to the case, so that the outputs' shapes do.
      same    all as the case says
      ragged  between half and all; of four sequences and more one place is free (its token gives zeros), one has no rows yet
      mixed   rows as in ragged; every eighth sequence brings all the new tokens, the others one"""
    n, new, B, kind = case["rows"], case["new"], case["B"], case["kind"]
    if kind == "same":
        return [n] * B, [new] * B
    g = torch.Generator()
    g.manual_seed(1000 * n + 10 * new + B)
    some = lambda top: [int(x) for x in torch.randint(top // 2, top + 1, (B,), generator=g)]  # noqa: E731
    rows, news = some(n), [max(x, 1) for x in some(new)]
    rows[0], news[0] = n, new
    if kind == "mixed":
        news = [new if b % 8 == 0 else 1 for b in range(B)]
    if B >= 4:
        rows[B // 2], news[B // 2] = -1, 1
        rows[B - 1] = 0
    return rows, news


def _states(case):
    """The two states of a planned batch, each as (rows that stay, new tokens): the second starts from less than the first one ends with, as
    after an eviction, and where a batch is mixed some sequences end and others take their places."""
    rows, news = _layout(case)
    cut = [max(r * 3 // 4, 0) if r >= 0 else 0 for r in rows]
    if case["kind"] == "mixed":
        cut = [-1 if b % 5 == 4 else r for b, r in enumerate(cut)]
    if case["kind"] == "same" and case["new"] == 1:  # generation, where a page in so many is full
        rows = [r + b % case["page"] for b, r in enumerate(rows)]
        cut = [r + 1 for r in rows]
    return (rows, news), (cut, [1] * case["B"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    order = lambda n: torch.randperm(n, generator=gen, device="cuda").to(torch.int32)  # noqa: E731
    return {"plan": _prepare_plan, "rotary": _prepare_rotary, "chunk": _prepare_chunk}[case["op"]](case, randn, ints, order, gen)


def _prepare_plan(case, randn, ints, order, gen):
    B, page = case["B"], case["page"]
    states = _states(case)
    ends = [[max(r, 0) + n for r, n in zip(*st)] for st in states]
    # before the first pass the batch holds what the second state ends with
    held = [-(-e // page) if r >= 0 else 0 for r, e in zip(states[1][0], ends[1])]
    need = max(sum(-(-e // page) for r, e in zip(st[0], end) if r >= 0) for st, end in zip(states, ends))
    N = max(need, sum(held)) + 5 if not case["tight"] else max(sum(held), need * 9 // 10) + 1
    most = max(-(-e // page) for end in ends for e in end) + 1
    pages, table = order(N), torch.full((B, most), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at:at + n]
        at += n
    free = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    free[:N - at] = pages[at:]
    T = max(sum(st[1]) for st in states) + 3
    base = torch.randint(0, 5000, (B,), generator=gen, device="cuda", dtype=torch.int32)
    return dict(case=case, turn=0, table=table, held=ints(held), free=free, n_free=ints([N - at]),
                len=[ints(st[0]) for st in states], new=[ints(st[1]) for st in states], seen=[ints(st[0]).clamp(min=0) + base for st in states],
                start=ints([0] * B), len_after=ints([0] * B), seen_after=ints([0] * B), token_start=ints([0] * (B + 1)),
                rows=torch.zeros(T, dtype=torch.int64, device="cuda"), pos=ints([0] * T))


def _prepare_rotary(case, randn, ints, order, gen):
    T, H, Hkv, D, page, dt = case["T"], case["H"], case["Hkv"], case["D"], case["page"], DTYPES[case["dtype"]]
    N = -(-T // page) + 3
    qkv = randn(T, (H + 2 * Hkv) * D).to(dt)  # one projection's output, whose parts are views
    q, k, v = qkv[:, :H * D].view(T, H, D), qkv[:, H * D:(H + Hkv) * D].view(T, Hkv, D), qkv[:, (H + Hkv) * D:].view(T, Hkv, D)
    # tokens lie in pages in runs, as sequences' do
    slot = torch.arange(T, device="cuda")
    rows = order(N)[slot // page].long() * page + slot % page
    if case["pad"]:
        rows[T - case["pad"]:] = -1  # a padded batch
    first = torch.randint(0, max(case["last"] - T, 1), (), generator=gen, device="cuda")
    pos = (first + torch.arange(T, device="cuda")).to(torch.int32)
    freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]) / case["factor"]
    pool = lambda: randn(N, Hkv, page, D).to(dt)  # noqa: E731
    return dict(case=case, q=q, k=k, v=v, rows=rows, pos=pos, freq=freq.float(), mscale=0.1 * math.log(case["factor"]) + 1.0, q_out=torch.zeros((T, H, D), dtype=dt, device="cuda"),
                k_pages=pool(), v_pages=pool(), pos_pages=torch.zeros((N, 1, page), dtype=torch.int32, device="cuda"),
                mass_pages=torch.ones((N, 1, page), device="cuda"))


def _prepare_chunk(case, randn, ints, order, gen):
    H, Hkv, D, page, dt = case["H"], case["Hkv"], case["D"], case["page"], DTYPES[case["dtype"]]
    rows, news = _layout(case)
    used = [-(-(r + n) // page) if r >= 0 else 0 for r, n in zip(rows, news)]
    N, most, T = sum(used) + 3, max(used) + 1, sum(news) + (0 if case["kind"] == "same" else 3)
    pages, table = order(N), torch.full((case["B"], most), -1, dtype=torch.int32, device="cuda")
    at, starts = 0, [0]
    for b, n in enumerate(used):
        table[b, :n] = pages[at:at + n]
        at += n
        starts.append(starts[-1] + news[b])
    # a twentieth of the keys draw much attention, the others little, as in prompts
    gain = torch.where(torch.rand((N, 1, page, 1), generator=gen, device="cuda") < 0.05, 4.0, 0.7)
    s = dict(case=case, table=table, start=ints(rows), token_start=ints(starts), k=(randn(N, Hkv, page, D) * gain).to(dt), v=randn(N, Hkv, page, D).to(dt),
             q=randn(T, H, D).to(dt), out=torch.zeros((T, H, D), dtype=dt, device="cuda"), lse=None)
    if case["lse"]:
        s["lse"] = torch.zeros((T, H), device="cuda")
    if own:
        from paper_2407_18121_amd import binding as ec
        s["ws"] = ec.new_workspace(ec.EC_FN_PAGED_CHUNK_STEP, case["B"], H, T, D, ec.dtype_code(s["q"]))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    op, case = s["case"]["op"], s["case"]
    if op == "plan":
        i = s["turn"]
        s["turn"] = 1 - i
        (_own_plan if own else _plain_plan)(s, s["len"][i], s["new"][i], s["seen"][i])
        return {k: s[k] for k in ("table", "held", "free", "n_free", "start", "len_after", "seen_after", "token_start", "rows", "pos")}
    if op == "rotary":
        if own:
            from paper_2407_18121_amd import binding as ec
            ec.ec_paged_rotary_store(s["q"], s["k"], s["v"], s["pos"], s["rows"], s["freq"], s["q_out"], s["k_pages"], s["v_pages"], s["pos_pages"],
                                     s["mass_pages"], interleaved=case["interleaved"], mscale=s["mscale"])
        else:
            _plain_rotary(s)
        return {k: s[k] for k in ("q_out", "k_pages", "v_pages", "pos_pages", "mass_pages")}
    if own:
        from paper_2407_18121_amd import binding as ec
        ec.ec_paged_chunk_step(s["q"], s["k"], s["v"], s["table"], s["start"], s["token_start"], case["D"] ** -0.5, s["out"], s["ws"], lse=s["lse"])
    else:
        _plain_chunk(s)
    return {"out": s["out"], **({"lse": s["lse"]} if case["lse"] else {})}


def _own_plan(s, length, new, seen):
    from paper_2407_18121_amd import binding as ec
    ec.ec_paged_plan(length, new, s["table"], s["held"], s["free"], s["n_free"], s["case"]["page"], s["start"], s["len_after"], s["token_start"],
                     s["rows"], s["pos"], seen_b=seen, seen_after_b=s["seen_after"])


# ------------------------------------------------------------------ the plain form
def _plain_plan(s, length, new, seen):
    page, table, T = s["case"]["page"], s["table"], s["rows"].shape[0]
    dev, most = table.device, table.shape[1]
    L, n, held = length.long(), new.long().clamp(min=0), s["held"].long()
    live = L >= 0
    ends = n.cumsum(0)
    want, keep = (torch.where(live, (x + page - 1) // page, 0) for x in (L + n, L))
    fits = live & (ends <= T) & (want <= most)
    goal = torch.where(fits, want, keep)
    gives, asks = (held - goal).clamp(min=0), torch.where(fits, goal - held, 0).clamp(min=0)
    n_free = s["n_free"].long()
    there = n_free + gives.sum()
    granted = fits & ((asks == 0) | (asks.cumsum(0) <= there))
    takes = torch.where(granted, asks, 0)
    entry = torch.arange(most, device=dev)
    # given back from a sequence's last page on, sequence after sequence: the entries of the reversed rows in order
    b, e = ((entry < held[:, None]) & (entry >= (held - gives)[:, None])).flip(1).nonzero(as_tuple=True)
    e = most - 1 - e
    s["free"][n_free + torch.arange(b.shape[0], device=dev)] = table[b, e]
    table[b, e] = -1
    b, e = ((entry >= held[:, None]) & (entry < (held + takes)[:, None])).nonzero(as_tuple=True)
    table[b, e] = s["free"][there - 1 - torch.arange(b.shape[0], device=dev)]
    s["held"].copy_(held - gives + takes)
    s["n_free"].copy_(there - b.shape[0])
    s["start"].copy_(torch.where(granted, L, -1))
    s["len_after"].copy_(torch.where(live, L + torch.where(granted, n, 0), -1))
    s["seen_after"].copy_(seen.long() + torch.where(granted, n, 0))
    s["token_start"][0] = 0
    s["token_start"][1:] = ends.clamp(max=T)
    t = torch.arange(T, device=dev)
    b = torch.searchsorted(ends, t, right=True)
    real = b < L.shape[0]
    b = b.clamp(max=L.shape[0] - 1)
    i = t - (ends - n)[b]
    real &= granted[b]
    slot = torch.where(real, L[b] + i, 0)
    s["rows"].copy_(torch.where(real, table[b, slot // page].long() * page + slot % page, -1))
    s["pos"].copy_(torch.where(real, seen.long()[b] + i, 0))


def _plain_rotary(s):
    case = s["case"]
    rot, page = case["rot"], case["page"]
    live = (s["rows"] >= 0).nonzero()[:, 0]
    angle = s["pos"][live].double()[:, None] * s["freq"].double()
    cos, sin = (f(angle).float()[:, None] * s["mscale"] for f in (torch.cos, torch.sin))

    def turned(x):
        y = x[live].float()
        if case["interleaved"]:
            a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
            y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()
            y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
        return y.to(x.dtype)

    p, o = s["rows"][live] // page, s["rows"][live] % page
    s["q_out"][live] = turned(s["q"])
    s["k_pages"][p, :, o] = turned(s["k"])
    s["v_pages"][p, :, o] = s["v"][live]
    s["pos_pages"][p, :, o] = s["pos"][live][:, None]
    s["mass_pages"][p, :, o] = 0.0


def _plain_chunk(s):
    case = s["case"]
    H, Hkv, D, page = case["H"], case["Hkv"], case["D"], case["page"]
    group, dev = H // Hkv, s["q"].device
    rows, news = _layout(case)
    at = 0
    for b, (L, n) in enumerate(zip(rows, news)):
        mine = slice(at, at + n)
        at += n
        if L < 0:
            s["out"][mine] = 0
            if case["lse"]:
                s["lse"][mine] = -math.inf
            continue
        ids = s["table"][b, :-(-(L + n) // page)].long()
        hidden = torch.arange(L + n, device=dev) > L + torch.arange(n, device=dev)[:, None]  # rows behind the token's own
        q = s["q"][mine].float().view(n, Hkv, group, D)
        at_once = max(1, min(Hkv, (1 << 30) // (n * group * (L + n))))  # key/value heads
        for h in range(0, Hkv, at_once):
            k, v = (x[ids, h:h + at_once].float().transpose(0, 1).reshape(-1, ids.shape[0] * page, D)[:, :L + n] for x in (s["k"], s["v"]))
            x = torch.matmul(q[:, h:h + at_once].permute(1, 2, 0, 3).reshape(k.shape[0], group * n, D), k.transpose(1, 2)) * D ** -0.5
            x = x.view(-1, group, n, L + n).masked_fill_(hidden, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - top)
            total = e.sum(-1, keepdim=True)
            y = torch.matmul((e / total).view(-1, group * n, L + n), v).view(-1, group, n, D)
            s["out"][mine].view(n, Hkv, group, D)[:, h:h + at_once] = y.permute(2, 0, 1, 3)
            if case["lse"]:
                s["lse"][mine].view(n, Hkv, group)[:, h:h + at_once] = (top + torch.log(total))[..., 0].permute(2, 0, 1)


# ------------------------------------------------------------------ what it costs, and what it is
def work(case):
    if case["op"] == "plan":
        (rows, news), (cut, ones) = _states(case)
        page, T = case["page"], max(sum(news), sum(ones)) + 3
        ends = [[-(-(r + n) // page) if r >= 0 else 0 for r, n in zip(*st)] for st in ((rows, news), (cut, ones))]
        moved = sum(abs(x - y) for x, y in zip(*ends))
        tokens = (sum(news) + sum(ones)) / 2
        return {"bytes": 4 * case["B"] * 9 + 16 * moved + 12 * T + 4 * tokens / page, "flops": 0}
    e, D, H, Hkv = 4 if case["dtype"] == "f32" else 2, case["D"], case["H"], case["Hkv"]
    if case["op"] == "rotary":
        n = case["T"] - case["pad"]
        return {"bytes": n * (2 * (H + 2 * Hkv) * D * e + 12 + 8) + 8 * case["pad"], "flops": 3 * n * (H + Hkv) * case["rot"]}
    live = [(L, n) for L, n in zip(*_layout(case)) if L >= 0]
    seen = sum(n * L + n * (n + 1) // 2 for L, n in live)  # rows that the tokens see
    tokens = sum(n for _, n in live)
    return {"bytes": sum(L + n for L, n in live) * 2 * Hkv * D * e + tokens * 2 * H * D * e + (4 * tokens * H if case["lse"] else 0), "flops": 4 * seen * H * D}


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "rotary": _exact_rotary, "chunk": _exact_chunk}[case["op"]](case, s)


def _exact_plan(case, s):
    page = case["page"]
    L, new, seen = (s[k][0].tolist() for k in ("len", "new", "seen"))
    table, held, free, n_free = s["table"].tolist(), s["held"].tolist(), s["free"].tolist(), s["n_free"].tolist()[0]
    T, most = len(s["rows"]), len(table[0])
    pages = lambda n: -(-n // page)  # noqa: E731
    starts, goals = [0], []
    for b, n in enumerate(new):
        starts.append(starts[-1] + n)
        fits = L[b] >= 0 and starts[-1] <= T and pages(L[b] + n) <= most
        goals.append(pages(L[b] + n) if fits else None)
        keep = goals[b] if fits else pages(max(L[b], 0))
        while held[b] > keep:
            held[b] -= 1
            free[n_free], table[b][held[b]] = table[b][held[b]], -1
            n_free += 1
    start, after, seen_after = [], [], []
    asked, there = 0, n_free
    for b, n in enumerate(new):
        more = max(goals[b] - held[b], 0) if goals[b] is not None else 0
        asked += more
        granted = goals[b] is not None and (more == 0 or asked <= there)
        for _ in range(more if granted else 0):
            n_free -= 1
            table[b][held[b]] = free[n_free]
            held[b] += 1
        start.append(L[b] if granted else -1)
        after.append(-1 if L[b] < 0 else L[b] + n if granted else L[b])
        seen_after.append(seen[b] + n if granted else seen[b])
    rows, pos = [-1] * T, [0] * T
    for b, n in enumerate(new):
        for i in range(n if start[b] >= 0 else 0):
            slot = start[b] + i
            rows[starts[b] + i], pos[starts[b] + i] = table[b][slot // page] * page + slot % page, seen[b] + i
    put = lambda like, x: torch.tensor(x, dtype=like.dtype, device=like.device)  # noqa: E731
    return {"table": put(s["table"], table), "held": put(s["held"], held), "free": put(s["free"], free), "n_free": put(s["n_free"], [n_free]),
            "start": put(s["start"], start), "len_after": put(s["len_after"], after), "seen_after": put(s["seen_after"], seen_after),
            "token_start": put(s["token_start"], [min(x, T) for x in starts]), "rows": put(s["rows"], rows), "pos": put(s["pos"], pos)}


def _exact_rotary(case, s):
    rot, page = case["rot"], case["page"]
    n = case["T"] - case["pad"]
    # element d of the turned part: its pair's other half, that half's sign, its frequency
    d = torch.arange(rot, device="cuda")
    other, sign, which = ((d ^ 1, d % 2 * 2 - 1, d // 2) if case["interleaved"] else ((d + rot // 2) % rot, torch.where(d < rot // 2, -1, 1), d % (rot // 2)))
    angle = torch.outer(s["pos"][:n].double(), s["freq"].double())[:, which]

    def turned(x):
        y = x[:n].double()
        z = y.clone()
        z[..., :rot] = s["mscale"] * (y[..., :rot] * torch.cos(angle)[:, None] + sign * y[..., other] * torch.sin(angle)[:, None])
        return z

    got = {name: s[name].double() for name in ("q_out", "k_pages", "v_pages", "mass_pages")}
    got["pos_pages"] = s["pos_pages"]
    page_of, in_page = s["rows"][:n] // page, s["rows"][:n] % page
    got["q_out"][:n] = turned(s["q"])
    got["k_pages"][page_of, :, in_page] = turned(s["k"])
    got["v_pages"][page_of, :, in_page] = s["v"][:n].double()
    got["pos_pages"][page_of, 0, in_page] = s["pos"][:n]
    got["mass_pages"][page_of, 0, in_page] = 0
    return got


def _exact_chunk(case, s):
    page, group = case["page"], case["H"] // case["Hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    table, L, first = s["table"].tolist(), s["start"].tolist(), s["token_start"].tolist()
    for b in range(case["B"]):
        t0, t1 = first[b], first[b + 1]
        if L[b] < 0:
            lse[t0:t1] = -math.inf
            continue
        slots = torch.arange(L[b] + t1 - t0, device="cuda")
        p = torch.tensor(table[b], device="cuda")[slots // page].long()
        for h in range(case["H"]):
            k, v = (x[p, h // group, slots % page].double() for x in (s["k"], s["v"]))
            for i in range(t0, t1, 512):
                j = min(i + 512, t1)
                sees = L[b] + j - t0
                x = (s["q"][i:j, h].double() @ k[:sees].T) / math.sqrt(case["D"])
                x = torch.where(slots[:sees] <= L[b] + torch.arange(i - t0, j - t0, device="cuda")[:, None], x, -math.inf)
                out[i:j, h] = torch.softmax(x, 1) @ v[:sees]
                lse[i:j, h] = torch.logsumexp(x, 1)
    return {"out": out, **({"lse": lse} if case["lse"] else {})}
