"""The paged key/value cache of the verification step: its operators, in plain form and through the library.

A round verifies a chunk of new tokens per request (the last emitted token and K drafts).  The forward pass in front of
it needs three operators around the paged cache of keys and values, and this file holds the cases they are timed and
compared on:

  plan       request lengths and the round's accepted lengths in; block tables, page moves and slot maps out
             (``binding.cache_plan``)
  append     the chunk's keys and values into their slots (``binding.cache_append``)
  attention  the chunk's queries over the cache (``binding.chunk_attention``)

``own`` False: elementary torch operations in 32 bits.  ``own`` True: the calls a user makes of the library.
"""
import math

import torch

own = False

NO_ROOM, NO_PAGES = 64, 128  # status bits of a plan, as in include/specsteer.h
BAD_LEN = 2

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    att = lambda name, **k: dict(op="attention", name=name, **k)  # noqa: E731
    return [
        # one user, one drafted block of four on a short conversation: the smallest call, where latency counts
        att("attention_one_request", B=1, n_lo=5, n_hi=5, past_lo=715, past_hi=715, Hq=16, Hkv=8, D=128, page=16, window=0, dtype="bf16"),
        # plain decoding, one token per request, ragged contexts down to nothing
        att("attention_single_tokens", B=64, n_lo=1, n_hi=1, past_lo=0, past_hi=4001, Hq=32, Hkv=8, D=64, page=32, window=0, dtype="f16"),
        # the batched verification shape (256 requests, four drafts each)
        att("attention_verify_batch", B=256, n_lo=5, n_hi=5, past_lo=130, past_hi=4000, Hq=64, Hkv=8, D=128, page=64, window=0, dtype="bf16"),
        # few requests with long private contexts: work has to be split along the cache
        att("attention_long_context", B=3, n_lo=9, n_hi=9, past_lo=30011, past_hi=120001, Hq=64, Hkv=8, D=128, page=128, window=0, dtype="bf16"),
        # layers that see a sliding window only; ragged draft lengths, some requests idle
        att("attention_window", B=64, n_lo=0, n_hi=7, past_lo=100, past_hi=9000, Hq=32, Hkv=4, D=128, page=16, window=1024, dtype="bf16"),
        # prompts taken in chunks on top of what is cached
        att("attention_prompt_chunks", B=4, n_lo=509, n_hi=2048, past_lo=0, past_hi=4099, Hq=32, Hkv=8, D=128, page=64, window=0, dtype="bf16"),
        # a whole long prompt in one call: bound by the tensor cores
        att("attention_long_prompt", B=1, n_lo=8192, n_hi=8192, past_lo=0, past_hi=0, Hq=32, Hkv=8, D=128, page=64, window=0, dtype="bf16"),
        # the plan of a round of one request, of a large batch, and of a step that takes prompts in
        dict(op="plan", name="plan_one_request", B=1, n_lo=5, n_hi=5, past_lo=715, past_hi=715, page=16, width=256),
        dict(op="plan", name="plan_large_batch", B=512, n_lo=7, n_hi=7, past_lo=0, past_hi=4001, page=16, width=512),
        dict(op="plan", name="plan_prompts", B=24, n_lo=1, n_hi=4096, past_lo=0, past_hi=9000, page=16, width=1024),
        # a verification chunk's keys and values, and a prompt step's
        dict(op="append", name="append_chunk", B=16, n_lo=6, n_hi=6, past_lo=100, past_hi=3000, Hkv=8, D=128, page=16, dtype="bf16"),
        dict(op="append", name="append_prompts", B=24, n_lo=100, n_hi=2500, past_lo=0, past_hi=1000, Hkv=8, D=128, page=64, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "plan", "append"))
    page = rng.choice((16, 32, 64, 128))
    if op == "plan":
        prompts = rng.random() < 0.4
        c = dict(op=op, B=_log_int(rng, 1, 64 if prompts else 700), n_lo=rng.randint(0, 3), n_hi=_log_int(rng, 16, 2000) if prompts else rng.randint(3, 9),
                 past_lo=rng.randint(0, 100), past_hi=_log_int(rng, 200, 7000), page=page, width=0)
        c["width"] = (c["past_hi"] + c["n_hi"] + 16) // page + 1 + rng.randint(0, 64)
        return c
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "append":
        prompts = rng.random() < 0.4
        return dict(op=op, B=_log_int(rng, 1, 24 if prompts else 500), n_lo=rng.randint(0, 3), n_hi=_log_int(rng, 16, 2000) if prompts else rng.randint(3, 9),
                    past_lo=0, past_hi=_log_int(rng, 10, 1000), Hkv=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 96, 128)), page=page, dtype=dtype)
    Hkv, D = rng.choice((1, 2, 4, 8)), rng.choice((64, 96, 128, 128))
    Hq = Hkv * rng.choice((1, 2, 4, 5, 6, 7, 8, 16) if Hkv < 8 else (1, 2, 4, 5, 8))
    prompts = rng.random() < 0.35
    window = rng.choice((0, 0, 0, rng.randint(1, 3000)))
    if prompts:
        B, n_hi, past_hi = _log_int(rng, 1, 6), _log_int(rng, 20, 4000), _log_int(rng, 1, 8000)
        n_lo = rng.randint(0, n_hi)
    else:
        B, past_hi = _log_int(rng, 1, 256), _log_int(rng, 16, 60000)
        n_hi = rng.randint(1, 9)
        n_lo = rng.randint(0, n_hi)
    c = dict(op=op, B=B, n_lo=n_lo, n_hi=n_hi, past_lo=rng.randint(0, past_hi), past_hi=past_hi, Hq=Hq, Hkv=Hkv, D=D, page=page, window=window, dtype=dtype)
    while True:  # no dearer than the largest listed cases: the cache, the plain form's scores, the products
        kv = c["past_hi"] + c["n_hi"]
        if c["B"] * kv * c["Hkv"] * c["D"] <= 1 << 30 and c["B"] * c["n_hi"] * kv * c["Hq"] <= 1 << 31 and work(c)["flops"] <= 5.4e11:
            return c
        if c["B"] > 1 and not prompts:
            c["B"] = (c["B"] + 1) // 2
        else:
            c["past_hi"], c["past_lo"], c["n_hi"], c["n_lo"] = c["past_hi"] * 3 // 4 + 1, c["past_lo"] * 3 // 4, c["n_hi"] * 3 // 4 + 1, c["n_lo"] * 3 // 4


def _lens(case):
    """(new tokens, tokens cached before them) per request: spread evenly over the ranges, the same for every seed.  The
    new tokens go up while the cached ones jump through their range."""
    B, got = case["B"], []
    for i in range(B):
        f, g = (i / (B - 1), ((i * 7919) % B) / (B - 1)) if B > 1 else (1.0, 1.0)
        got.append((case["n_lo"] + round((case["n_hi"] - case["n_lo"]) * f), case["past_lo"] + round((case["past_hi"] - case["past_lo"]) * g)))
    return got


def _keys(n, past, window):
    """(keys that some row sees, sum over the rows of the keys that each sees)."""
    if n == 0:
        return 0, 0
    if not window:
        return past + n, n * past + n * (n + 1) // 2
    seen = min(past + n, window + n - 1)
    full = max(0, min(n, past + n - window))  # rows whose window is full
    part = n - full
    return seen, full * window + part * past + part * (part + 1) // 2


def work(case):
    lens = _lens(case)
    T, page = sum(n for n, _ in lens), case["page"]
    if case["op"] == "plan":
        moved = sum((past + n + page - 1) // page - (past + page - 1) // page for n, past in lens)
        # per request four words in and out, per token a slot (8), a position (4), a request (4), per page moved a read and a write
        return {"bytes": 32 * case["B"] + 16 * T + 8 * moved, "flops": 0}
    if case["op"] == "append":
        return {"bytes": 2 * 2 * T * case["Hkv"] * case["D"] * 2 + 8 * T, "flops": 0}
    seen = [_keys(n, past, case["window"]) for n, past in lens]
    keys, pairs = sum(k for k, _ in seen), sum(p for _, p in seen)
    return {"bytes": keys * case["Hkv"] * case["D"] * 4 + T * case["Hq"] * (case["D"] * 4 + 4) + 4 * (keys // page + case["B"]),
            "flops": 4 * case["D"] * case["Hq"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _pool(lens, page, width, g, spare):
    """Pages of a pool handed out in random order: block table, pages in use, the pages left over."""
    dev = g.device
    kv = torch.tensor([n + past for n, past in lens], dtype=torch.int64, device=dev)
    pages = (kv + page - 1) // page
    total = sum((n + past + page - 1) // page for n, past in lens)
    order = torch.randperm(total + spare, generator=g, device=dev).to(torch.int32)
    first = torch.cumsum(pages, 0) - pages
    j = torch.arange(width, device=dev)
    at = (first[:, None] + j[None, :]).clamp_(max=total + spare - 1)
    table = torch.where(j[None, :] < pages[:, None], order[at], torch.full_like(at, -1, dtype=torch.int32))
    return table.contiguous(), pages, order[total:], total + spare


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed) + 1)
    B, page, lens = case["B"], case["page"], _lens(case)
    lens = [lens[i] for i in torch.randperm(B, generator=cpu).tolist()]
    T = sum(n for n, _ in lens)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"op": case["op"], "page": page, "T": T}
    if case["op"] == "plan":
        # the state after a round: the last chunk's drafts were kept in part (advance), a few requests are done (-1),
        # a few are new (nothing held); the pages of the last chunk are still held
        width = case["width"]
        last = [(0, 0) if past == 0 else (min(8, past), past - min(8, past)) for _, past in lens]
        used = [(n, past) for n, past in last]
        extra = sum((n + page) // page + 2 for n, _ in lens) + 7
        table, held, free, P = _pool([(n + min(8, past), past) for n, past in used], page, width, g, extra)
        new = [-1 if torch.rand((), generator=cpu).item() < 0.02 and B > 8 else n for n, _ in lens]
        adv = [int(torch.randint(0, n + 1, (), generator=cpu)) for n, _ in used]
        head = int(torch.randint(0, 1 << 40, (), generator=cpu))
        ring = torch.full((P,), -1, dtype=torch.int32, device=dev)
        ring[(head + torch.arange(free.numel(), device=dev)) % P] = free
        cap = T + 13
        s.update(seq_len=i32([past for _, past in used]), advance=i32(adv), new_len=i32(new), pages_held=held.to(torch.int32), block_table=table, free_ring=ring,
                 ring_pos=torch.tensor([head, head + free.numel()], dtype=torch.int64, device=dev), max_tokens=cap)
        # the program's buffers for what a plan says
        e = lambda n, dt=torch.int32: torch.empty(n, dtype=dt, device=dev)  # noqa: E731
        s["out"] = {"seq_len": e(B), "pages_held": e(B), "ring_pos": e(2, torch.int64), "cu_new": e(B + 1), "kv_len": e(B), "slot_map": e(cap, torch.int64),
                    "positions": e(cap), "token_req": e(cap), "status": e(B)}
        return s
    dt = DTYPES[case["dtype"]]
    width = max((n + past + page - 1) // page for n, past in lens) or 1
    table, _, _, P = _pool(lens, page, width, g, 3)
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev, dtype=dt)  # noqa: E731
    Hkv, D = case["Hkv"], case["D"]
    s.update(k_cache=randn(P, page, Hkv, D), v_cache=randn(P, page, Hkv, D))
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    if case["op"] == "append":
        slots = []
        t = table.cpu()
        for b, (n, past) in enumerate(lens):
            pos = torch.arange(past, past + n)
            slots.append(t[b][pos // page].to(torch.int64) * page + pos % page)
        pad = torch.full((5,), -1, dtype=torch.int64)  # a padded batch: rows behind the last token name no slot
        s.update(slot_map=torch.cat(slots + [pad]).to(dev), k=randn(T + 5, Hkv, D), v=randn(T + 5, Hkv, D))
        return s
    s.update(q=randn(T, case["Hq"], D), block_table=table, cu_new=i32(cu), kv_len=i32([n + past for n, past in lens]), window=case["window"],
             scale=1.0 / math.sqrt(D), n_max=max(n for n, _ in lens), kv_max=max(n + past for n, past in lens))
    s.update(out=torch.empty_like(s["q"]), lse=torch.empty(T, case["Hq"], dtype=torch.float32, device=dev))  # the program's buffers
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_plan(s):
    page, table, ring, cap = s["page"], s["block_table"], s["free_ring"], s["max_tokens"]
    B, W = table.shape
    P, dev = ring.numel(), table.device
    seq, new, held = s["seq_len"].long(), s["new_len"].long(), s["pages_held"].long()
    gone = new == -1
    kept = torch.where(gone, 0, seq + s["advance"].long())
    asked = new.clamp(min=0)
    bad = (new < -1) | (kept < 0) | (kept + asked > W * page) | (held < 0) | (held > W)
    asked = torch.where(bad, 0, asked)
    no_room = (torch.cumsum(asked, 0) > cap) & (asked > 0)
    asked = torch.where(no_room, 0, asked)
    target = torch.where(bad, held, (kept + asked + page - 1) // page)
    give, take = (held - target).clamp(min=0), (target - held).clamp(min=0)
    head, tail = s["ring_pos"][0], s["ring_pos"][1]
    given = torch.minimum(give.sum(), P - (tail - head))
    cum_give, cum_take = torch.cumsum(give, 0), torch.cumsum(take, 0)
    refused = (take > 0) & (cum_take > tail - head + given)
    asked, take = torch.where(refused, 0, asked), torch.where(refused, 0, take)
    held_out = torch.where(refused, held, target)
    # pages given back, in request order, behind the ring's tail
    r = torch.arange(P, device=dev)
    b = torch.searchsorted(cum_give, r, right=True).clamp(max=B - 1)
    page_of = table[b, (held_out[b] + r - (cum_give - give)[b]).clamp(0, W - 1)]
    at = (tail + r) % P
    ring[at] = torch.where(r < given, page_of, ring[at])
    # pages taken, in request order, from its head
    taken = take.sum()
    b = torch.searchsorted(torch.cumsum(take, 0), r, right=True).clamp(max=B - 1)
    j = (held[b] + r - (torch.cumsum(take, 0) - take)[b]).clamp(0, W - 1)
    live = r < taken
    table[b[live], j[live]] = ring[(head + r) % P][live]
    # the tokens of the next chunk
    cu = torch.zeros(B + 1, dtype=torch.int64, device=dev)
    cu[1:] = torch.cumsum(asked, 0)
    i = torch.arange(cap, device=dev)
    b = torch.searchsorted(cu[1:].contiguous(), i, right=True).clamp(max=B - 1)
    pos = kept[b] + i - cu[b]
    live = i < cu[B]
    slot = table[b, (pos // page).clamp(0, W - 1)].long() * page + pos % page
    i32 = torch.int32
    return {"seq_len": torch.where(bad, seq, kept).to(i32), "pages_held": held_out.to(i32), "ring_pos": torch.stack((head + taken, tail + given)),
            "cu_new": cu.to(i32), "kv_len": torch.where(bad, 0, kept + asked).to(i32), "slot_map": torch.where(live, slot, -1),
            "positions": torch.where(live, pos, -1).to(i32), "token_req": torch.where(live, b, -1).to(i32),
            "status": (bad * BAD_LEN + no_room * NO_ROOM + refused * NO_PAGES).to(i32), "block_table": table, "free_ring": ring}


def _plain_append(s):
    live = s["slot_map"] >= 0
    slot = s["slot_map"][live]
    for cache, x in (("k_cache", "k"), ("v_cache", "v")):
        s[cache].view(-1, *s[cache].shape[2:])[slot] = s[x][live]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    q, table, cu, kv_len, n_max, kv_max = s["q"], s["block_table"], s["cu_new"].long(), s["kv_len"].long(), s["n_max"], s["kv_max"]
    T, Hq, D = q.shape
    _, page, Hkv, _ = s["k_cache"].shape
    B, dev = table.shape[0], q.device
    W = (kv_max + page - 1) // page
    pages = table[:, :W].long().clamp(min=0)
    k = s["k_cache"][pages].reshape(B, W * page, Hkv, D).float().permute(0, 2, 3, 1)            # [B, Hkv, D, keys]
    v = s["v_cache"][pages].reshape(B, W * page, Hkv, D).float().permute(0, 2, 1, 3)            # [B, Hkv, keys, D]
    i = torch.arange(n_max, device=dev)
    n = cu[1:] - cu[:-1]
    row = (cu[:-1, None] + i[None, :]).clamp(max=T - 1)
    x = q[row].float().reshape(B, n_max, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    score = (x @ k).mul_(s["scale"]).view(B, Hkv, Hq // Hkv, n_max, W * page)
    pos = (kv_len - n)[:, None] + i[None, :]                                                    # position of each row
    j = torch.arange(W * page, device=dev)
    hidden = j[None, None, :] > pos[:, :, None]
    if s["window"]:
        hidden |= j[None, None, :] <= pos[:, :, None] - s["window"]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = (score.view(B, Hkv, -1, W * page) @ v).view(B, Hkv, Hq // Hkv, n_max, D) / total.clamp(min=1e-37)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    live = i[None, :] < n[:, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n_max, Hq, D)[live]
    lse = lse[..., 0].permute(0, 3, 1, 2).reshape(B, n_max, Hq)[live]
    return {"out": out.to(q.dtype), "lse": lse}


def run(s):
    if own:
        from paper_2603_16219_b200 import binding
        if s["op"] == "plan":
            got = binding.cache_plan(s["seq_len"], s["new_len"], s["pages_held"], s["block_table"], s["free_ring"], s["ring_pos"], page_size=s["page"],
                                     max_tokens=s["max_tokens"], advance=s["advance"], out=s["out"])
            return dict(got, block_table=s["block_table"], free_ring=s["free_ring"])
        if s["op"] == "append":
            binding.cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slot_map"])
            return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        out, lse = binding.chunk_attention(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["cu_new"], s["kv_len"], scale=s["scale"], window=s["window"],
                                           out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    return {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention}[s["op"]](s)


# ---- what the definitions say, in 64 bits ---------------------------------------------------------------------------
def _exact_plan(s):
    """Request by request, with lists."""
    page, cap = s["page"], s["max_tokens"]
    seq, adv, new, held = (s[k].tolist() for k in ("seq_len", "advance", "new_len", "pages_held"))
    table, ring = s["block_table"].tolist(), s["free_ring"].tolist()
    head, tail = s["ring_pos"].tolist()
    P, W, B = len(ring), len(table[0]), len(seq)
    status, kept, asked, first, total = [0] * B, [0] * B, [0] * B, list(held), 0
    for b in range(B):
        kept[b] = 0 if new[b] == -1 else seq[b] + adv[b]
        asked[b] = max(new[b], 0)
        if new[b] < -1 or kept[b] < 0 or kept[b] + asked[b] > W * page or not 0 <= held[b] <= W:
            status[b], asked[b] = BAD_LEN, 0
            continue
        total += asked[b]
        if asked[b] and total > cap:
            status[b], asked[b] = NO_ROOM, 0
        target = -(-(kept[b] + asked[b]) // page)
        for j in range(target, held[b]):
            if tail - head < P:
                ring[tail % P] = table[b][j]
                tail += 1
        first[b] = min(held[b], target)
    free, at = tail - head, head
    out = {k: [] for k in ("seq_len", "pages_held", "kv_len", "slot_map", "positions", "token_req")}
    cu, wanted = [0], 0
    for b in range(B):
        held_out = held[b]
        if status[b] != BAD_LEN:
            target = -(-(kept[b] + asked[b]) // page)
            more = target - first[b]
            wanted += more
            if more and wanted > free:
                status[b], asked[b] = status[b] | NO_PAGES, 0
            else:
                for j in range(first[b], target):
                    table[b][j] = ring[at % P]
                    at += 1
                held_out = target
        for i in range(asked[b]):
            p = kept[b] + i
            out["slot_map"].append(table[b][p // page] * page + p % page)
            out["positions"].append(p)
            out["token_req"].append(b)
        cu.append(cu[-1] + asked[b])
        out["seq_len"].append(seq[b] if status[b] == BAD_LEN else kept[b])
        out["kv_len"].append(0 if status[b] == BAD_LEN else kept[b] + asked[b])
        out["pages_held"].append(held_out)
    for k in ("slot_map", "positions", "token_req"):
        out[k] += [-1] * (cap - cu[-1])
    out.update(cu_new=cu, status=status, ring_pos=[at, tail], block_table=table, free_ring=ring)
    return {k: torch.tensor(v, dtype=torch.int64 if k in ("slot_map", "ring_pos") else torch.int32) for k, v in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "plan":
        return _exact_plan(s)
    if s["op"] == "append":
        slots, page = s["slot_map"].tolist(), s["page"]
        rows = [t for t, slot in enumerate(slots) if slot >= 0]
        pages, offs = [slots[t] // page for t in rows], [slots[t] % page for t in rows]
        caches = {}
        for cache, x in (("k_cache", "k"), ("v_cache", "v")):
            caches[cache] = s[cache].double()
            caches[cache][pages, offs] = s[x][rows].double()
        return caches
    q, scale, window = s["q"], s["scale"], s["window"]
    T, Hq, D = q.shape
    Hkv, page = s["k_cache"].shape[2], s["page"]
    G = Hq // Hkv
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    cu, kv = s["cu_new"].tolist(), s["kv_len"].tolist()
    for b in range(len(kv)):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        pages = s["block_table"][b, :-(-kv[b] // page)].long()
        ks, vs = (s[c][pages].flatten(0, 1)[:kv[b]].double() for c in ("k_cache", "v_cache"))
        for r0 in range(0, n, 1024):
            rows = torch.arange(r0, min(n, r0 + 1024), device=q.device)
            pos = kv[b] - n + rows
            lo, hi = max(0, kv[b] - n + r0 - window + 1) if window else 0, kv[b] - n + int(rows[-1]) + 1
            keys = torch.arange(lo, hi, device=q.device)
            seen = keys[None, :] <= pos[:, None]
            if window:
                seen &= keys[None, :] > pos[:, None] - window
            for h in range(Hkv):
                x = q[cu[b] + r0:cu[b] + r0 + len(rows), h * G:(h + 1) * G].double() * scale                # [rows, G, D]
                score = torch.einsum("rgd,kd->grk", x, ks[lo:hi, h]).masked_fill(~seen, -math.inf)
                z = torch.logsumexp(score, -1)
                o = torch.exp(score - z[..., None]) @ vs[lo:hi, h]
                out[cu[b] + r0:cu[b] + r0 + len(rows), h * G:(h + 1) * G] = o.transpose(0, 1)
                lse[cu[b] + r0:cu[b] + r0 + len(rows), h * G:(h + 1) * G] = z.transpose(0, 1)
    return {"out": out, "lse": lse}
