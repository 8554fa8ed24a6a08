"""Plain references of the operators of a round over trees of drafts, in float64 or with lists."""
import math

import numpy as np
import torch

MAX_ROWS = 1024


def random_parents(rng, n, kind="tree"):
    """Parents of n rows; the first hangs on the cache."""
    if n == 0:
        return []
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "forest":   # rows that hang on the cache alone among them
        return [-1] + [int(rng.integers(-1, i)) for i in range(1, n)]
    return [-1] + [int(rng.integers(max(0, (i - 1) // 4), i)) for i in range(1, n)]


def climb(parent, i):
    way = [i]
    while parent[way[-1]] >= 0:
        way.append(parent[way[-1]])
    return way


def plan_reference(parent, cu, kv, T, words, window=0):
    """(mask, positions, status): what is not written is None in positions."""
    mask = np.zeros((T, words), np.int64)
    pos, status = [None] * T, [0] * len(kv)
    accepted = [cu[b + 1] for b in range(len(kv)) if 0 <= cu[b] <= cu[b + 1] <= T and kv[b] >= cu[b + 1] - cu[b]]
    for t in range(max([0, cu[-1]] + accepted), T):
        pos[t] = -1
    for b in range(len(kv)):
        n = cu[b + 1] - cu[b]
        if cu[b] < 0 or n < 0 or cu[b + 1] > T or kv[b] < n:
            status[b] |= 2
            continue
        if n > min(MAX_ROWS, 32 * words):
            status[b] |= 2
            for t in range(cu[b], cu[b + 1]):
                pos[t] = -1
            continue
        p = list(parent[cu[b]:cu[b + 1]])
        for i in range(n):
            if not -1 <= p[i] < i:
                p[i] = -1
                status[b] |= 1024
        for i in range(n):
            way = climb(p, i)
            pos[cu[b] + i] = kv[b] - n + len(way) - 1
            for j in way[:window or None]:
                mask[cu[b] + i, j // 32] |= 1 << (j % 32)
    return np.where(mask >= 1 << 31, mask - (1 << 32), mask).astype(np.int32), pos, status


def pack_bits(seen, words):
    """[n, n] of truth values as [n, words] int32."""
    n = seen.shape[0]
    bits = np.zeros((n, words * 32), np.int64)
    bits[:, :n] = seen
    packed = (bits.reshape(n, words, 32) << np.arange(32)).sum(-1)
    return np.where(packed >= 1 << 31, packed - (1 << 32), packed).astype(np.int32)


def attention_reference(q, k_cache, v_cache, table, cu, kv_len, mask, scale, window=0, positions=None):
    """(out, lse, bound of out, bound of lse, written) in float64; the bounds count the roundings as _paged.attention_reference does."""
    T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_cache.shape
    G = Hq // Hkv
    u, e = torch.finfo(q.dtype).eps / 2, 2.0 ** -24
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    tol_o, tol_l, written = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros(T, bool)
    qd, kd, vd = (x.double().cpu().numpy() for x in (q, k_cache, v_cache))
    tb, bits = table.cpu().numpy(), mask.cpu().numpy().astype(np.int64) & 0xffffffff
    words = bits.shape[1]
    for b in range(len(kv_len)):
        n, kv = cu[b + 1] - cu[b], kv_len[b]
        if cu[b] < 0 or n < 0 or cu[b + 1] > T or kv < n or kv > tb.shape[1] * page or n > 32 * words:
            continue
        past = kv - n
        for i in range(n):
            row = cu[b] + i
            written[row] = True
            lo = 0
            if window:
                lo = max(0, min(max(int(positions[row]), past), past + i) - window + 1)
            j = np.array([x for x in range(lo, past)] + [past + x for x in range(n) if bits[row, x // 32] >> (x % 32) & 1], np.int64)
            if len(j) == 0:
                continue
            pages = tb[b, j // page]
            ok = (pages >= 0) & (pages < n_pages)
            j, pages = j[ok], pages[ok]
            if len(j) == 0:
                continue
            k, v = kd[pages, j % page], vd[pages, j % page]
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
                    f16 = q.dtype == torch.float16
                    tiny = len(j) * 2.0 ** -25 * np.abs(v[:, h // G]).max(0) if f16 else 0.0
                    tol_l[row, h] = err + len(j) * e + 4 * e * abs(lse[row, h])
                    tol_o[row, h] = A * (u * (1 + u) + 2 * err + 2 * len(j) * e + 2.0 ** -20) + np.abs(out[row, h]) * u + tiny + (2.0 ** -25 if f16 else 0.0)
    return out, lse, tol_o, tol_l, written


def rotate_reference(x, weight, eps, positions, inv_freq, axis_of, neighbours, factor):
    """(heads normed and turned, bound) in float64.  x [T, H, D], positions [axes, T] lists.

    The bound, with e = 2^-24 and S = |x w| + |x' w'|, both normed, times the factor: an angle is a number of turns below 1/2 rounded to
    float32 (2^-26, times 2 pi: 2^-23.3) and its sine and cosine are off by 2^-23 more (2^-22.1 together, doubled for what the roundings of pi
    in the formula add); of a far position the number of turns carries 1.5 half steps of float64 beside (the reference forms the same
    product); a norm by D/2 e for the sum, 2^-22.9 for the root and 2 e; the products and their sum by 6 e."""
    T, H, D = x.shape
    u, e = torch.finfo(x.dtype).eps / 2, 2.0 ** -24
    x = x.double().cpu()
    half = len(inv_freq)
    if eps is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if weight is not None:
            x = x * weight.double().cpu()
    f = inv_freq.double().cpu().tolist()
    angle = torch.zeros(T, half, dtype=torch.float64)
    for i in range(half):
        a = 0 if axis_of is None else axis_of[i]
        if 0 <= a < len(positions):
            angle[:, i] = torch.tensor(positions[a], dtype=torch.float64) * f[i]
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y, size = x.clone(), x.abs()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if neighbours else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = factor * (a * c - b * s), factor * (b * c + a * s)
    size[..., first] = size[..., second] = abs(factor) * (a.abs() + b.abs())
    far = angle.abs().max(1).values[:, None, None] * 1.5 * 2.0 ** -53 if half else 0.0
    bound = size * (2.0 ** -21.1 + far + 2.0 ** -22.9 + (D / 2 + 10) * e)
    floor = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}[{2.0 ** -11: torch.float16, 2.0 ** -8: torch.bfloat16, 2.0 ** -24: torch.float32}[u]]
    return y, bound + u * (y.abs() + bound) + floor


def logprobs_reference(x, temperature=None):
    """(log probabilities [R, V], lse, entropy, bounds of lse, of entropy and, but for 6 e of its own size, of a log probability) in float64.

    With e = 2^-24 and d = |l - max l|: a weight is off by 2^-22 and 5 e d relative (the difference, c and the product are rounded); its
    share of a sum by one e for every addition on its way, fewer than 256 (36 in a tile, one a tile, the warp's and the rows' joining)."""
    x = x.double().cpu()
    e = 2.0 ** -24
    l = x if temperature is None else x / temperature.double().cpu()[:, None]
    logp = torch.log_softmax(l, 1)
    p = logp.exp()
    m = l.max(1, keepdim=True).values
    d = torch.where(p > 0, m - l, torch.zeros_like(l))
    mean = (p * d).sum(1)
    lse = torch.logsumexp(l, 1)
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    s = 256 * e + 2.0 ** -22 + 5 * e * mean                       # of the sum, relative
    tol_lse = s + 4 * e * (lse.abs() + m[:, 0].abs()) + 2.0 ** -22
    spread = (p * d * d).sum(1)
    tol_h = s + (256 * e + 2.0 ** -22) * (1 + mean) + 6 * e * (spread + mean) + s * mean + 2.0 ** -22
    return logp, lse, entropy, tol_lse, tol_h, s + 2.0 ** -22 + 6 * e * (lse - m[:, 0])


def top_reference(x, k):
    """Ids of the k largest of every row, the lowest among equals."""
    return torch.sort(x.double().cpu(), dim=1, descending=True, stable=True).indices[:, :k]


def keep_reference(parent, token, choice, cu, kv, T, max_out, table=None, page=0, n_pages=0):
    """(n_out, path, out_tokens, moves [(request, from slot, to slot)], status) with lists."""
    n_out, path, toks, moves, status = [], [], [], [], []
    for b in range(len(kv)):
        n = cu[b + 1] - cu[b]
        bad = cu[b] < 0 or n < 0 or cu[b + 1] > T or kv[b] < n or n > MAX_ROWS or (table is not None and kv[b] > table.shape[1] * page)
        st, way = (2 if bad else 0), []
        if not bad and n > 0:
            way = [0]
            while len(way) < max_out:
                kids = [i for i in range(way[-1] + 1, n) if parent[cu[b] + i] == way[-1] and token[cu[b] + i] == choice[cu[b] + way[-1]] >= 0]
                if not kids:
                    break
                way.append(kids[0])
        if table is not None:
            for i, j in enumerate(way):
                if i == j:
                    continue
                src, dst = kv[b] - n + j, kv[b] - n + i
                ps, pd = int(table[b, src // page]), int(table[b, dst // page])
                if 0 <= ps < n_pages and 0 <= pd < n_pages:
                    moves.append((ps * page + src % page, pd * page + dst % page))
                else:
                    st |= 32
        n_out.append(len(way))
        path.append(way + [-1] * (max_out - len(way)))
        toks.append([choice[cu[b] + i] for i in way] + [-1] * (max_out - len(way)))
        status.append(st)
    return n_out, path, toks, moves, status
