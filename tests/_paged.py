"""Plain references of the paged cache's operators: float64 attention request by request, the plan with lists."""
import math

import numpy as np
import torch

BAD_LEN, BAD_PAGE, NO_ROOM, NO_PAGES, BAD_POOL = 2, 32, 64, 128, 256


def plan_reference(seq_len, advance, new_len, held, table, ring, ring_pos, page, max_tokens, n_pages):
    """The plan as specsteer_cache_plan defines it, one request after the other.  Lists in, a dict of arrays out."""
    B, W = len(seq_len), table.shape[1]
    table, ring = table.copy(), ring.copy()
    head, tail = ring_pos
    pool_ok = head >= 0 and 0 <= tail - head <= n_pages
    status, kept, asked, target = [0] * B, [0] * B, [0] * B, [0] * B
    total = 0
    for b in range(B):
        n = new_len[b]
        kept[b] = 0 if n == -1 else seq_len[b] + advance[b]
        asked[b] = max(n, 0)
        if n < -1 or kept[b] < 0 or kept[b] + asked[b] > min(W * page, 2 ** 31 - 1) or not 0 <= held[b] <= W:
            status[b] |= BAD_LEN
        if not pool_ok:
            status[b] |= BAD_POOL
        if status[b]:
            asked[b], target[b] = 0, held[b]
            continue
        total += asked[b]
        if asked[b] and total > max_tokens:
            status[b] |= NO_ROOM
            asked[b] = 0
        target[b] = -(-(kept[b] + asked[b]) // page)
        for j in range(target[b], held[b]):
            if tail - head < n_pages:
                ring[tail % n_pages] = table[b, j]
                tail += 1
    wanted, front = 0, head
    held_out = list(target)
    for b in range(B):
        if status[b] & (BAD_LEN | BAD_POOL) or target[b] <= held[b]:
            continue
        wanted += target[b] - held[b]
        if wanted > tail - head:
            status[b] |= NO_PAGES
            asked[b], held_out[b] = 0, held[b]
        else:
            for j in range(held[b], target[b]):
                table[b, j] = ring[front % n_pages]
                front += 1
    cu = [0]
    slot, pos, req = [], [], []
    for b in range(B):
        for i in range(asked[b]):
            p = kept[b] + i
            pg = int(table[b, p // page])
            ok = 0 <= pg < n_pages
            if not ok:
                status[b] |= BAD_PAGE
            slot.append(pg * page + p % page if ok else -1)
            pos.append(p)
            req.append(b)
        cu.append(len(slot))
    pad = [-1] * (max_tokens - len(slot))
    refused = [bool(s & (BAD_LEN | BAD_POOL)) for s in status]
    return {"seq_len": [seq_len[b] if refused[b] else kept[b] for b in range(B)], "pages_held": held_out, "ring_pos": [front, tail] if pool_ok else list(ring_pos),
            "cu_new": cu, "kv_len": [0 if refused[b] else kept[b] + asked[b] for b in range(B)], "slot_map": slot + pad, "positions": pos + pad,
            "token_req": req + pad, "status": status, "block_table": table, "free_ring": ring}


def attention_reference(q, k_cache, v_cache, table, cu, kv_len, scale, window=0):
    """(out, lse, bound of out, bound of lse, written) in float64 on the CPU.  Only the keys that a row sees are touched.

    The bounds count every rounding of the kernels, with u = half a step of the inputs' type and e = 2^-24:
      scores      (D + 2) e sum_d |q_d k_d| scale absolute (float32 accumulation in any order, the multiplication by scale)
      weights     2^(.) to 2^-21 relative, its argument to 4 e |argument| absolute: both relative errors of the weight
      rounding    u relative per weight for the product with v; F16 weights below 2^-14 to 2^-25 absolute against a sum >= 1
      sums        n e relative over n keys
      result      u relative, and 2^-20 for the division and the joining of parts
    """
    T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_cache.shape
    G = Hq // Hkv
    u, e = torch.finfo(q.dtype).eps / 2, 2.0 ** -24
    out = np.zeros((T, Hq, D))
    lse = np.full((T, Hq), -np.inf)
    tol_o, tol_l = np.zeros((T, Hq, D)), np.zeros((T, Hq))
    written = np.zeros(T, bool)
    qd = q.double().cpu().numpy()
    kd, vd = k_cache.double().cpu().numpy(), v_cache.double().cpu().numpy()
    tb = table.cpu().numpy()
    for b in range(len(kv_len)):
        n, kv = cu[b + 1] - cu[b], kv_len[b]
        if cu[b] < 0 or n < 0 or cu[b + 1] > T or kv < 0 or kv > tb.shape[1] * page:
            continue
        for i in range(n):
            row = cu[b] + i
            written[row] = True
            hi = kv - n + i + 1
            lo = max(0, hi - window) if window else 0
            j = np.arange(lo, max(lo, hi))
            pages = tb[b, j // page]
            ok = (pages >= 0) & (pages < n_pages)
            j, pages = j[ok], pages[ok]
            if len(j) == 0:
                continue
            k = kd[pages, j % page]                 # [keys, Hkv, D]
            v = vd[pages, j % page]
            for h in range(Hq):
                x = qd[row, h]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = (k[:, h // G] @ x) * scale
                    m = s.max()
                    w = np.exp(s - m)
                    l = w.sum()
                    out[row, h] = (w @ v[:, h // G]) / l
                    lse[row, h] = m + math.log(l) if np.isfinite(l) and l > 0 else (np.nan if np.isnan(l) else m)
                    size = np.abs(k[:, h // G]) @ np.abs(x) * scale
                    err = ((D + 2) * e * size + 8 * e * (np.abs(s) + abs(m) + 12) + 2.0 ** -21).max()
                    A = (w @ np.abs(v[:, h // G])) / l
                    tiny = len(j) * 2.0 ** -25 * np.abs(v[:, h // G]).max(0) if q.dtype == torch.float16 else 0.0
                    tol_l[row, h] = err + len(j) * e + 4 * e * abs(lse[row, h])
                    tol_o[row, h] = A * (u * (1 + u) + 2 * err + 2 * len(j) * e + 2.0 ** -20) + np.abs(out[row, h]) * u + tiny + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
    return out, lse, tol_o, tol_l, written


def build_cache(lens, page, Hkv, D, dtype, device, seed, layout="nhd", width_extra=0, spare=2):
    """Random pools with the pages of every request handed out in random order; slots nobody uses hold NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-kv // page) for _, kv in lens]
    P = sum(need) + spare
    perm = torch.randperm(P, generator=g)
    W = max(need + [1]) + width_extra
    table = torch.full((len(lens), W), -7, dtype=torch.int32)
    used = torch.zeros(P, page, dtype=torch.bool)
    at = 0
    for b, (_, kv) in enumerate(lens):
        table[b, :need[b]] = perm[at:at + need[b]].to(torch.int32)
        for i in range(need[b]):
            used[perm[at + i], :min(page, kv - i * page)] = True
        at += need[b]
    caches = []
    for _ in range(2):
        c = torch.randn(P, page, Hkv, D, generator=g).to(dtype)
        c[~used] = float("nan")
        if layout == "hnd":
            c = c.permute(0, 2, 1, 3).contiguous().to(device).permute(0, 2, 1, 3)
        elif layout == "joined":                       # keys and values of a page side by side in one pool
            c = c.to(device)
        else:
            c = c.to(device)
        caches.append(c)
    if layout == "joined":
        pool = torch.stack(caches, 1).contiguous()
        caches = [pool[:, 0], pool[:, 1]]
    T = sum(n for n, _ in lens)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    return caches[0], caches[1], table.to(device), cu, [kv for _, kv in lens], T, g
