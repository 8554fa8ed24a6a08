"""A round over trees of drafts, and the probabilities of its tokens: operators in plain form and through the library.

A request may draft a tree of tokens instead of a chain: row 0 of its chunk is the last emitted token, and every other row
names its parent.  The forward pass of such a chunk, and what follows it, need five operators, and this file holds the
cases they are timed and compared on:

  plan       parents in; the ancestors of every row as bits, and its position out          (``binding.tree_plan``)
  rotate     queries and keys normed by head and turned by their positions (of one axis or several, as for images and
             video), keys and values into their slots of the paged cache, in one pass      (``binding.rotate_append``)
  attention  every row over the cache and over its ancestors                               (``binding.tree_attention``)
  logprobs   log probabilities of given tokens, entropy, the likeliest tokens of a row     (``binding.token_logprobs``)
  keep       the path of drafts that the tokens chosen behind each row confirm, and its keys and values moved together
             in the cache of every layer                                                   (``binding.tree_keep``)

``own`` False: elementary torch operations, in 32 bits (angles in 64).  ``own`` True: the calls a user makes of the library.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    att = lambda name, **k: dict(op="attention", name=name, **k)  # noqa: E731
    return [
        # one user, a small tree on a short conversation: latency counts
        att("attention_one_request", B=1, n_lo=9, n_hi=9, past_lo=715, past_hi=715, Hq=16, Hkv=8, D=128, page=16, window=0, dtype="bf16"),
        # a batch of verification rounds with trees of up to 32 nodes over ragged contexts
        att("attention_batch", B=64, n_lo=15, n_hi=32, past_lo=130, past_hi=4000, Hq=64, Hkv=8, D=128, page=64, window=0, dtype="bf16"),
        # wide trees on long private contexts: work has to be split along the cache
        att("attention_long_context", B=2, n_lo=49, n_hi=63, past_lo=30011, past_hi=120001, Hq=32, Hkv=8, D=128, page=128, window=0, dtype="bf16"),
        # layers that see a sliding window only; narrow heads, ragged trees, some requests idle
        att("attention_window", B=48, n_lo=0, n_hi=25, past_lo=100, past_hi=9000, Hq=32, Hkv=4, D=64, page=16, window=1024, dtype="f16"),
        # the tree of one request, and of a large batch
        dict(op="plan", name="plan_one_request", B=1, n_lo=9, n_hi=9, past_lo=715, past_hi=715, words=1, window=0),
        dict(op="plan", name="plan_batch", B=256, n_lo=3, n_hi=200, past_lo=0, past_hi=4001, words=8, window=0),
        # a verification batch's chunk (256 requests, five rows each), one axis of positions
        dict(op="rotate", name="rotate_chunk", B=256, n_lo=5, n_hi=5, past_lo=130, past_hi=4000, Hq=64, Hkv=8, D=128, rot=128, axes=1, neighbours=False, norm=True,
             page=64, dtype="bf16"),
        # prompts with images in them: positions along time, height and width
        dict(op="rotate", name="rotate_images", B=6, n_lo=509, n_hi=2048, past_lo=0, past_hi=30001, Hq=32, Hkv=8, D=128, rot=128, axes=3, neighbours=False, norm=True,
             page=64, dtype="bf16"),
        # the rows of one request; those of a verification batch over a large vocabulary, with what an interface shows of each token
        dict(op="logprobs", name="logprobs_one_request", R=5, V=32000, M=1, top=8, tempered=False, dtype="f32"),
        dict(op="logprobs", name="logprobs_batch", R=1280, V=151936, M=1, top=20, tempered=True, dtype="bf16"),
        # the path of one request in a cache of 36 layers; of a batch in one of 16
        dict(op="keep", name="keep_one_request", B=1, n_lo=9, n_hi=9, past_lo=715, past_hi=715, layers=36, Hkv=8, D=128, page=16, max_out=6, dtype="bf16"),
        dict(op="keep", name="keep_batch", B=64, n_lo=15, n_hi=32, past_lo=0, past_hi=300, layers=16, Hkv=8, D=128, page=16, max_out=8, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "plan", "rotate", "logprobs", "logprobs", "keep"))
    if op == "logprobs":
        c = dict(op=op, R=_log_int(rng, 1, 1500), V=_log_int(rng, 900, 256000), M=rng.choice((1, 1, 2, 5)), top=rng.choice((0, 1, 5, 8, 20, 32)),
                 tempered=rng.random() < 0.5, dtype=rng.choice(("bf16", "bf16", "f32", "f16")))
        while c["R"] * c["V"] * SIZE[c["dtype"]] > 388 * 10 ** 6:
            c["R"] = (c["R"] + 1) // 2
        return c
    if op == "plan":
        n_hi = _log_int(rng, 2, 1000)
        c = dict(op=op, B=_log_int(rng, 1, 500), n_lo=rng.randint(0, n_hi), n_hi=n_hi, past_lo=rng.randint(0, 100), past_hi=_log_int(rng, 200, 7000), words=0,
                 window=rng.choice((0, 0, rng.randint(1, 9))))
        while c["B"] > 1 and c["B"] * c["n_hi"] ** 2 > 256 * 200 ** 2:
            c["B"] = (c["B"] + 1) // 2
        c["words"] = (n_hi + 31) // 32 + rng.choice((0, 0, 1))
        return c
    page, dtype = rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "bf16", "f16"))
    if op == "rotate":
        D = rng.choice((64, 80, 96, 128, 128, 256))
        prompts = rng.random() < 0.4
        n_hi = _log_int(rng, 16, 2000) if prompts else rng.randint(1, 30)
        return dict(op=op, B=_log_int(rng, 1, 6 if prompts else 80), n_lo=rng.randint(0, n_hi // 2 + 1), n_hi=n_hi, past_lo=0, past_hi=_log_int(rng, 10, 60000),
                    Hq=rng.choice((4, 7, 16, 32)), Hkv=rng.choice((1, 2, 4)), D=D, rot=rng.choice((D, D, D // 2)), axes=rng.choice((1, 1, 2, 3)),
                    neighbours=rng.random() < 0.4, norm=rng.random() < 0.7, page=page, dtype=rng.choice((dtype, dtype, "f32")))
    if op == "keep":
        n_hi = rng.randint(1, 60)
        return dict(op=op, B=_log_int(rng, 1, 64), n_lo=rng.randint(0, n_hi), n_hi=n_hi, past_lo=0, past_hi=_log_int(rng, 10, 300), layers=rng.choice((1, 3, 8, 16)),
                    Hkv=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 96, 128)), page=page, max_out=rng.randint(2, 9), dtype=dtype)
    Hkv, D = rng.choice((1, 2, 4, 8)), rng.choice((64, 96, 128, 128))
    Hq = Hkv * rng.choice((1, 2, 4, 5, 6, 7, 8, 16) if Hkv < 8 else (1, 2, 4, 5, 8))
    n_hi, past_hi = _log_int(rng, 2, 200), _log_int(rng, 16, 60000)
    c = dict(op=op, B=_log_int(rng, 1, 200), n_lo=rng.randint(0, n_hi), n_hi=n_hi, past_lo=rng.randint(0, past_hi), past_hi=past_hi, Hq=Hq, Hkv=Hkv, D=D, page=page,
             window=rng.choice((0, 0, 0, rng.randint(1, 3000))), dtype=dtype)
    while True:  # no dearer than the largest listed cases: the cache, the plain form's scores, the products
        kv = c["past_hi"] + c["n_hi"]
        if c["B"] * kv * c["Hkv"] * c["D"] <= 1 << 28 and c["B"] * c["n_hi"] * kv * c["Hq"] <= 1 << 29 and work(c)["flops"] <= 1.5e11:
            return c
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        else:
            c["past_hi"], c["past_lo"], c["n_hi"], c["n_lo"] = c["past_hi"] * 3 // 4 + 1, c["past_lo"] * 3 // 4, c["n_hi"] * 3 // 4 + 1, c["n_lo"] * 3 // 4


def _lens(case):
    """(rows, tokens cached before them) per request: spread evenly over the ranges, the same for every seed.  The rows go
    up while the cached tokens jump through their range."""
    B, got = case["B"], []
    for i in range(B):
        f, g = (i / (B - 1), ((i * 7919) % B) / (B - 1)) if B > 1 else (1.0, 1.0)
        got.append((case["n_lo"] + round((case["n_hi"] - case["n_lo"]) * f), case["past_lo"] + round((case["past_hi"] - case["past_lo"]) * g)))
    return got


def _depth(n):
    """About how many rows a path of such a tree has (parents are drawn between a quarter and a half of a row's number)."""
    return 1 + int(math.log(n, 3)) if n > 1 else n


def work(case):
    op = case["op"]
    if op == "logprobs":
        R, V = case["R"], case["V"]
        return {"bytes": R * V * SIZE[case["dtype"]] + R * (8 * case["M"] + 8 * case["top"] + 8 + 4 * case["tempered"]), "flops": 5 * R * V}
    lens = _lens(case)
    T = sum(n for n, _ in lens)
    if op == "plan":
        return {"bytes": T * (8 + 4 * case["words"]) + 8 * case["B"], "flops": 0}
    es = SIZE[case["dtype"]]
    if op == "rotate":
        heads = case["Hq"] + case["Hkv"]
        return {"bytes": 2 * T * (heads + case["Hkv"]) * case["D"] * es + T * (8 + 4 * case["axes"]), "flops": T * heads * case["D"] * (3 + 4 * case["norm"])}
    if op == "keep":
        moved = sum(min(_depth(n), case["max_out"]) // 2 for n, _ in lens)
        return {"bytes": 2 * 2 * moved * case["layers"] * case["Hkv"] * case["D"] * es + 12 * T + 8 * case["B"] * (case["max_out"] + 2), "flops": 0}
    seen = [(min(past, case["window"] - 1) if case["window"] else past) for _, past in lens]
    pairs = sum(n * (s + _depth(n)) for (n, _), s in zip(lens, seen))
    keys = sum(s + n for (n, _), s in zip(lens, seen) if n)
    return {"bytes": keys * case["Hkv"] * case["D"] * 2 * es + T * case["Hq"] * (case["D"] * 2 * es + 4) + 4 * (keys // case["page"] + case["B"]),
            "flops": 4 * case["D"] * case["Hq"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _trees(lens, cpu):
    """Parents of every row: the first row of a request hangs on its cache, the others on a row between a quarter and a
    half of their own number."""
    got = []
    for n, _ in lens:
        i = torch.arange(n)
        lo, hi = (i - 1).clamp(min=0) // 4, (i - 1).clamp(min=0) // 2
        p = lo + (torch.rand(n, generator=cpu) * (hi - lo + 1)).long()
        p[:1] = -1
        got.append(torch.minimum(p, (i - 1).clamp(min=-1)))
    return got


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed) + 1)
    op = case["op"]
    s = {"op": op}
    randn = lambda *shape, dt: torch.randn(*shape, generator=g, device=dev, dtype=dt)  # noqa: E731
    empty = lambda *shape, dt: torch.empty(*shape, device=dev, dtype=dt)  # noqa: E731
    f32, i32 = torch.float32, torch.int32
    if op == "logprobs":
        R, V, M, top = case["R"], case["V"], case["M"], case["top"]
        x = randn(R, V, dt=DTYPES[case["dtype"]]).mul_(2.5)
        x.scatter_add_(1, torch.randint(0, V, (R, 8), generator=g, device=dev), (torch.rand(R, 8, generator=g, device=dev) * 14).to(x.dtype))  # a few likely tokens
        s.update(logits=x, tokens=torch.randint(0, V, (R, M), generator=g, device=dev, dtype=i32), top=top,
                 temperature=torch.rand(R, generator=g, device=dev) * 1.5 + 0.25 if case["tempered"] else None)
        s["out"] = {"lse": empty(R, dt=f32), "entropy": empty(R, dt=f32), "logprob": empty(R, M, dt=f32), "top_id": empty(R, top, dt=i32), "top_logprob": empty(R, top, dt=f32)}
        return s
    B, lens = case["B"], _lens(case)
    lens = [lens[i] for i in torch.randperm(B, generator=cpu).tolist()]
    T, pad = sum(n for n, _ in lens), 3  # a padded batch: three rows behind the last request's
    cu = torch.zeros(B + 1, dtype=torch.int64)
    cu[1:] = torch.cumsum(torch.tensor([n for n, _ in lens]), 0)
    s.update(cu_new=cu.to(i32).to(dev), kv_len=torch.tensor([n + past for n, past in lens], dtype=i32, device=dev), n_max=max(n for n, _ in lens))
    n_of = torch.tensor([n for n, _ in lens])
    req, row = torch.repeat_interleave(torch.arange(B), n_of), torch.arange(T) - torch.repeat_interleave(cu[:-1], n_of)  # request of each row, its number there
    past = torch.tensor([p for _, p in lens])
    if op != "rotate":
        parent = torch.cat(_trees(lens, cpu) + [torch.full((pad,), -1)])
        s["parent"] = parent.to(i32).to(dev)
    if op == "plan":
        s.update(words=case["words"], window=case["window"])
        s["out"] = {"mask": empty(T + pad, case["words"], dt=i32), "positions": empty(T + pad, dt=i32)}
        return s
    dt, page, Hkv, D = DTYPES[case["dtype"]], case["page"], case["Hkv"], case["D"]
    # pages handed out in random order
    pages = [(n + p + page - 1) // page for n, p in lens]
    P = sum(pages) + 3
    order, width, first = torch.randperm(P, generator=cpu), max(pages) or 1, 0
    table = torch.full((B, width), -1, dtype=torch.int64)
    for b, m in enumerate(pages):
        table[b, :m] = order[first:first + m]
        first += m
    s["block_table"] = table.to(i32).to(dev)
    cache = ((case["layers"],) if op == "keep" else ()) + (P, page, Hkv, D)
    s.update(k_cache=randn(*cache, dt=dt), v_cache=randn(*cache, dt=dt))
    if op == "keep":
        # the tokens of a tree, and the token that the verification chose behind each row: mostly one of the row's children
        token = torch.randint(0, 50, (T + pad,), generator=cpu)
        choice = torch.randint(0, 50, (T + pad,), generator=cpu)
        kids = torch.nonzero(parent[:T] >= 0).flatten()
        kids = kids[torch.rand(kids.numel(), generator=cpu) < 0.8]
        choice[cu[req[kids]] + parent[kids]] = token[kids]
        s.update(token=token.to(i32).to(dev), choice=choice.to(i32).to(dev), max_out=case["max_out"])
        s["out"] = {"n_out": empty(B, dt=i32), "path": empty(B, case["max_out"], dt=i32), "out_tokens": empty(B, case["max_out"], dt=i32)}
        return s
    Hq = case["Hq"]
    if op == "rotate":
        at = past[req] + row
        slot = torch.cat([table[req, at // page] * page + at % page, torch.full((pad,), -1)])
        axes = case["axes"]
        pos = at[None].repeat(axes, 1)
        if axes > 1:  # half of the rows are patches of pictures: their time stands still while height and width run
            side = 17
            picture = (at // 289) % 2 == 1
            for a in range(axes):
                run = at // 289 * side if a == 0 else at // 289 * side + (at % 289 // side if a == 1 else at % side)
                pos[a] = torch.where(picture, run, pos[a])
        qkv = randn(T + pad, Hq + 2 * Hkv, D, dt=dt)  # what one projection leaves
        half = case["rot"] // 2
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], slot_map=slot.to(dev), positions=torch.cat([pos, torch.full((axes, pad), -1)], 1).to(i32).to(dev),
                 inv_freq=(1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(dev), neighbours=case["neighbours"], eps=1e-6 if case["norm"] else None,
                 axis_of=(torch.arange(half) * axes // half).to(i32).to(dev) if axes > 1 else None)
        s["weights"] = [1 + 0.1 * randn(D, dt=f32) for _ in range(2)] if case["norm"] else [None, None]
        s["q_out"] = torch.empty(T + pad, Hq, D, device=dev, dtype=dt)
        return s
    # attention: the plan's outputs stand for what a program has from the round's plan
    plan = _plain_plan(dict(s, words=max(1, (s["n_max"] + 31) // 32), window=case["window"]))
    s.update(q=randn(T + pad, Hq, D, dt=dt), mask=plan["mask"], positions=plan["positions"], window=case["window"], scale=1.0 / math.sqrt(D),
             kv_max=max(n + p for n, p in lens), rows=T)
    s.update(out=torch.zeros_like(s["q"]), lse=torch.zeros(T + pad, Hq, dtype=f32, device=dev))
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _rows(s, T):
    """Request and number of every row, and whether it is of a request at all."""
    cu = s["cu_new"].long()
    i = torch.arange(T, device=cu.device)
    req = torch.searchsorted(cu[1:].contiguous(), i, right=True).clamp(max=cu.numel() - 2)
    return req, i - cu[req], i < cu[-1]


def _above(parent, req, row, live, B, n_max):
    """[B, n, n]: whether j is i or an ancestor of i, by squaring the relation to the parent."""
    n = max(1, n_max)
    up = torch.eye(n, device=parent.device).repeat(B, 1, 1)
    has = live & (parent >= 0)
    up[req[has], row[has], parent[has].long()] = 1
    for _ in range((n - 1).bit_length()):
        up = (up @ up).clamp_(max=1)
    return up


def _plain_plan(s):
    T, words = s["parent"].numel(), s["words"]
    req, row, live = _rows(s, T)
    past = s["kv_len"].long() - (s["cu_new"][1:] - s["cu_new"][:-1]).long()
    up = _above(s["parent"], req, row, live, past.numel(), s["n_max"])
    depth = up.sum(-1) - 1                                                                      # [B, n]
    if s["window"]:
        up = up * (depth[:, None, :] > depth[:, :, None] - s["window"])
    bits = torch.zeros(past.numel(), up.shape[1], words * 32, device=up.device, dtype=torch.int64)
    bits[:, :, :up.shape[2]] = up.long()
    packed = (bits.view(past.numel(), up.shape[1], words, 32) << torch.arange(32, device=up.device)).sum(-1)
    packed = torch.where(packed >= 1 << 31, packed - (1 << 32), packed)
    at = row.clamp(max=up.shape[1] - 1)
    mask = torch.where(live[:, None], packed[req, at], 0)
    return {"mask": mask.to(torch.int32), "positions": torch.where(live, past[req] + depth[req, at].long(), -1).to(torch.int32)}


def _turned(x, weight, s):
    x = x.float()
    if s["eps"] is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight
    half = s["inv_freq"].numel()
    pos = s["positions"][0][:, None] if s["axis_of"] is None else s["positions"][s["axis_of"].long()].T   # [T, 1 or half]
    angle = pos.double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["neighbours"] else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_rotate(s):
    live = s["slot_map"] >= 0
    slot = s["slot_map"][live]
    k = _turned(s["k"], s["weights"][1], s).to(s["k"].dtype)
    for cache, x in (("k_cache", k), ("v_cache", s["v"])):
        s[cache].view(-1, *s[cache].shape[2:])[slot] = x[live]
    return {"q": _turned(s["q"], s["weights"][0], s).to(s["q"].dtype), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    q, table, cu, kv_len, n_max, kv_max = s["q"], s["block_table"], s["cu_new"].long(), s["kv_len"].long(), max(1, s["n_max"]), s["kv_max"]
    T, Hq, D = q.shape
    _, page, Hkv, _ = s["k_cache"].shape
    B, dev = table.shape[0], q.device
    W = max(1, (kv_max + page - 1) // page)
    pages = table[:, :W].long().clamp(min=0)
    k = s["k_cache"][pages].reshape(B, W * page, Hkv, D).float().permute(0, 2, 3, 1)            # [B, Hkv, D, keys]
    v = s["v_cache"][pages].reshape(B, W * page, Hkv, D).float().permute(0, 2, 1, 3)            # [B, Hkv, keys, D]
    i = torch.arange(n_max, device=dev)
    n = cu[1:] - cu[:-1]
    row = (cu[:-1, None] + i[None, :]).clamp(max=T - 1)
    x = q[row].float().reshape(B, n_max, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    score = (x @ k).mul_(s["scale"]).view(B, Hkv, Hq // Hkv, n_max, W * page)
    # a row sees the tokens in front of the chunk (within the window) and those of the chunk that its bits name
    past = kv_len - n
    j = torch.arange(W * page, device=dev)
    seen = (j[None, None, :] < past[:, None, None]).expand(B, n_max, -1)
    if s["window"]:
        seen = seen & (j[None, None, :] > s["positions"][row].long()[:, :, None] - s["window"])
    at = j[None, None, :] - past[:, None, None]                                                 # number of the key in the chunk
    words = s["mask"][row].long()                                                               # [B, n, words]
    bit = torch.gather(words, 2, (at >> 5).clamp(0, words.shape[2] - 1).expand(B, n_max, -1)) >> (at & 31) & 1
    seen = seen | ((at >= 0) & (at < n[:, None, None]) & (bit > 0))
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = (score.view(B, Hkv, -1, W * page) @ v).view(B, Hkv, Hq // Hkv, n_max, D) / total.clamp(min=1e-37)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    live = i[None, :] < n[:, None]
    s["out"][:s["rows"]] = out.permute(0, 3, 1, 2, 4).reshape(B, n_max, Hq, D)[live].to(q.dtype)
    s["lse"][:s["rows"]] = lse[..., 0].permute(0, 3, 1, 2).reshape(B, n_max, Hq)[live]
    return {"out": s["out"], "lse": s["lse"]}


def _plain_logprobs(s):
    x = s["logits"].float()
    # the order of the tokens: by logit, the lowest id among equals; keys of 64 bits hold both
    top = {}
    if s["top"]:
        bits = (x + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
        best = torch.topk(key, s["top"], dim=1).values
        top["top_id"] = (x.shape[1] - 1 - (best & 0xffffffff)).to(torch.int32)
        del key, bits
    if s["temperature"] is not None:
        x = x / s["temperature"][:, None]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    entropy = total.log() - (e * (x - m)).sum(1, keepdim=True) / total
    got = {"lse": lse[:, 0], "entropy": entropy[:, 0], "logprob": x.gather(1, s["tokens"].long()) - lse}
    if s["top"]:
        got.update(top, top_logprob=x.gather(1, top["top_id"].long()) - lse)
    return got


def _plain_keep(s):
    T, L, dev = s["parent"].numel(), s["max_out"], s["parent"].device
    req, row, live = _rows(s, T)
    cu = s["cu_new"].long()
    n, past = cu[1:] - cu[:-1], s["kv_len"].long() - (cu[1:] - cu[:-1])
    B, m = past.numel(), max(1, s["n_max"])
    # a row is confirmed when its token was chosen behind its parent and no sibling before it has the same token
    put = lambda x, fill: torch.full((B, m), fill, dtype=torch.int64, device=dev).index_put_((req[live], row[live]), x[live].long())  # noqa: E731
    parent, token, choice = put(s["parent"], -2), put(s["token"], -1), put(s["choice"], -1)
    ok = (parent >= 0) & (token == choice.gather(1, parent.clamp(min=0)))
    i = torch.arange(m, device=dev)
    twin = (parent[:, :, None] == parent[:, None, :]) & (token[:, :, None] == token[:, None, :]) & (i[None, None, :] < i[None, :, None])
    ok &= ~twin.any(-1)
    ok[:, 0] = n > 0
    up = _above(s["parent"], req, row, live, B, s["n_max"])
    on = ok & (up @ (~ok).float()[..., None] == 0)[..., 0] & (up[:, :, 0] > 0)                  # every row from the first to this one
    order = torch.where(on, i, m).sort(1).values                                                # paths run down the numbers
    path = torch.full((B, L), -1, dtype=torch.int64, device=dev)
    w = min(L, m)
    path[:, :w] = torch.where(order[:, :w] < m, order[:, :w], -1)
    out_tokens = torch.where(path >= 0, choice.gather(1, path.clamp(min=0)), -1)
    # the keys and values of the path, to the places behind the cached ones
    table, page = s["block_table"].long(), s["k_cache"].shape[2]
    to = torch.arange(L, device=dev)[None, :].expand(B, L)
    b, j = torch.nonzero((path >= 0) & (path != to), as_tuple=True)
    src, dst = past[b] + path[b, j], past[b] + j
    src, dst = table[b, src // page] * page + src % page, table[b, dst // page] * page + dst % page
    for cache in ("k_cache", "v_cache"):
        flat = s[cache].flatten(1, 2)
        flat[:, dst] = flat[:, src]
    return {"n_out": (path >= 0).sum(1).to(torch.int32), "path": path.to(torch.int32), "out_tokens": out_tokens.to(torch.int32), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(s):
    if own:
        from paper_2603_16219_b200 import binding
        if s["op"] == "plan":
            return binding.tree_plan(s["parent"], s["cu_new"], s["kv_len"], words=s["words"], window=s["window"], out=s["out"])
        if s["op"] == "rotate":
            q = binding.rotate_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["k_cache"], s["v_cache"], s["slot_map"], q_weight=s["weights"][0],
                                      k_weight=s["weights"][1], eps=s["eps"], axis_of=s["axis_of"], neighbours=s["neighbours"], q_out=s["q_out"])
            return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        if s["op"] == "attention":
            out, lse = binding.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["cu_new"], s["kv_len"], s["mask"], positions=s["positions"],
                                              scale=s["scale"], window=s["window"], out=s["out"], lse=s["lse"])
            return {"out": out, "lse": lse}
        if s["op"] == "logprobs":
            got = binding.token_logprobs(s["logits"], s["tokens"], temperature=s["temperature"], top=s["top"], out=s["out"])
            return got if s["top"] else {k: got[k] for k in ("lse", "entropy", "logprob")}
        got = binding.tree_keep(s["parent"], s["token"], s["choice"], s["cu_new"], s["kv_len"], s["block_table"], s["k_cache"], s["v_cache"], max_out=s["max_out"], out=s["out"])
        return dict(got, k_cache=s["k_cache"], v_cache=s["v_cache"])
    return {"plan": _plain_plan, "rotate": _plain_rotate, "attention": _plain_attention, "logprobs": _plain_logprobs, "keep": _plain_keep}[s["op"]](s)


# ---- what the definitions say, in 64 bits ---------------------------------------------------------------------------
def _climb(parent, n):
    """The rows from each row up to its root, by walking."""
    got = []
    for i in range(n):
        way, j = [], i
        while j >= 0:
            way.append(j)
            j = parent[j]
        got.append(way)
    return got


def _exact_plan(s):
    parent, cu, kv = s["parent"].tolist(), s["cu_new"].tolist(), s["kv_len"].tolist()
    mask = [[0] * s["words"] for _ in parent]
    pos = [-1] * len(parent)
    for b in range(len(kv)):
        n = cu[b + 1] - cu[b]
        for i, way in enumerate(_climb(parent[cu[b]:cu[b + 1]], n)):
            pos[cu[b] + i] = kv[b] - n + len(way) - 1
            for j in way[:s["window"] or None]:
                mask[cu[b] + i][j // 32] |= 1 << j % 32
    mask = [[w - (1 << 32) if w >> 31 else w for w in r] for r in mask]
    return {"mask": torch.tensor(mask, dtype=torch.int32), "positions": torch.tensor(pos, dtype=torch.int32)}


def _exact_rotate(s):
    def turned(x, weight):
        x = x.double()
        if s["eps"] is not None:
            x = x / ((x * x).mean(-1, keepdim=True) + s["eps"]).sqrt() * weight.double()
        freq = s["inv_freq"].double()
        half = freq.numel()
        axis = [0] * half if s["axis_of"] is None else s["axis_of"].tolist()
        angle = torch.stack([s["positions"][a].double() * freq[i] for i, a in enumerate(axis)], -1)[:, None]
        turn = torch.polar(torch.ones_like(angle), angle)                                       # each pair as a complex number
        r = x[..., :2 * half]
        z = torch.view_as_complex(r.reshape(*r.shape[:-1], half, 2).contiguous()) if s["neighbours"] else torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous())
        z = z * turn
        r = torch.view_as_real(z).flatten(-2) if s["neighbours"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([r, x[..., 2 * half:]], -1)

    rows = [t for t, slot in enumerate(s["slot_map"].tolist()) if slot >= 0]
    slots = s["slot_map"][rows]
    page = s["k_cache"].shape[1]
    got = {"q": turned(s["q"], s["weights"][0])}
    for cache, x in (("k_cache", turned(s["k"], s["weights"][1])), ("v_cache", s["v"].double())):
        got[cache] = s[cache].double()
        got[cache][slots // page, slots % page] = x[rows]
    return got


def _exact_attention(s):
    q, scale, window = s["q"], s["scale"], s["window"]
    T, Hq, D = q.shape
    Hkv, page = s["k_cache"].shape[2], s["k_cache"].shape[1]
    G, dev = Hq // Hkv, q.device
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=dev)
    lse = torch.zeros(T, Hq, dtype=torch.float64, device=dev)
    cu, kv, parent = s["cu_new"].tolist(), s["kv_len"].tolist(), s["parent"].tolist()
    for b in range(len(kv)):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        past = kv[b] - n
        pages = s["block_table"][b, :-(-kv[b] // page)].long()
        ks, vs = (s[c][pages].flatten(0, 1)[:kv[b]].double() for c in ("k_cache", "v_cache"))
        seen = torch.zeros(n, kv[b], dtype=torch.bool)
        for i, way in enumerate(_climb(parent[cu[b]:cu[b + 1]], n)):
            p = past + len(way) - 1
            seen[i, max(0, p - window + 1) if window else 0:past] = True
            seen[i, [past + j for j in way[:window or None]]] = True
        seen = seen.to(dev)
        for h in range(Hkv):
            x = q[cu[b]:cu[b + 1], h * G:(h + 1) * G].double() * scale                          # [rows, G, D]
            score = torch.einsum("rgd,kd->grk", x, ks[:, h]).masked_fill(~seen, -math.inf)
            z = torch.logsumexp(score, -1)
            out[cu[b]:cu[b + 1], h * G:(h + 1) * G] = (torch.exp(score - z[..., None]) @ vs[:, h]).transpose(0, 1)
            lse[cu[b]:cu[b + 1], h * G:(h + 1) * G] = z.transpose(0, 1)
    return {"out": out, "lse": lse}


def _exact_logprobs(s):
    R, V = s["logits"].shape
    got = {k: [] for k in ("lse", "entropy", "logprob", "top_id", "top_logprob")}
    for r0 in range(0, R, 128):
        raw = s["logits"][r0:r0 + 128].double()
        x = raw if s["temperature"] is None else raw / s["temperature"][r0:r0 + 128, None].double()
        logp = torch.log_softmax(x, 1)
        got["lse"].append(torch.logsumexp(x, 1))
        got["entropy"].append(-(logp.exp() * logp).sum(1))
        got["logprob"].append(logp.gather(1, s["tokens"][r0:r0 + 128].long()))
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :s["top"]]
        got["top_id"].append(order.to(torch.int32))
        got["top_logprob"].append(logp.gather(1, order))
    return {k: torch.cat(v) for k, v in got.items() if s["top"] or not k.startswith("top")}


def _exact_keep(s):
    parent, token, choice, cu, kv = (s[k].tolist() for k in ("parent", "token", "choice", "cu_new", "kv_len"))
    table, page, L = s["block_table"].tolist(), s["k_cache"].shape[2], s["max_out"]
    caches = {c: s[c].double() for c in ("k_cache", "v_cache")}
    n_out, paths, tokens = [], [], []
    for b in range(len(kv)):
        r0, n = cu[b], cu[b + 1] - cu[b]
        path = [0] if n else []
        while n and len(path) < L:
            kids = [i for i in range(n) if parent[r0 + i] == path[-1] and token[r0 + i] == choice[r0 + path[-1]]]
            if not kids:
                break
            path.append(kids[0])
        at = lambda p: (table[b][p // page], p % page)  # noqa: E731
        for i, j in enumerate(path):
            if i != j:
                (p0, o0), (p1, o1) = at(kv[b] - n + j), at(kv[b] - n + i)
                for c in caches.values():
                    c[:, p1, o1] = c[:, p0, o0]
        n_out.append(len(path))
        paths.append(path + [-1] * (L - len(path)))
        tokens.append([choice[r0 + i] for i in path] + [-1] * (L - len(path)))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return dict(caches, n_out=i32(n_out), path=i32(paths), out_tokens=i32(tokens))


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "rotate": _exact_rotate, "attention": _exact_attention, "logprobs": _exact_logprobs, "keep": _exact_keep}[case["op"]](s)
