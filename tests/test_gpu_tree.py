"""A round over trees of drafts on the GPU: each operator against its definition (tests/_tree.py), and a run of them together."""
import math

import numpy as np
import pytest
import torch

import _paged
import _tree
from _paged import BAD_LEN, BAD_PAGE, build_cache

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- plan -----------------------------------------------------------------------------------------------------------
def _check_plan(binding, parent, cu, kv, T, words, window=0, ld=None):
    wide = torch.full((T, ld or words), 77, dtype=torch.int32, device="cuda")
    out = {"mask": wide[:, :words], "positions": i32([77] * T)}
    status = i32([0] * len(kv))
    binding.tree_plan(i32(parent), i32(cu), i32(kv), words=words, window=window, out=out, status=status)
    mask, pos, want = _tree.plan_reference(parent, cu, kv, T, words, window)
    assert status.tolist() == want
    got_mask, got_pos = out["mask"].cpu().numpy(), out["positions"].tolist()
    for t in range(T):
        if pos[t] is None:
            assert got_pos[t] == 77 and (got_mask[t] == 77).all(), t
        else:
            assert got_pos[t] == pos[t] and (got_mask[t] == mask[t]).all(), t
    assert (wide[:, words:] == 77).all()


@pytest.mark.parametrize("B,n_hi,words,window,kind", [(1, 1, 1, 0, "tree"), (1, 9, 1, 0, "tree"), (7, 33, 2, 0, "tree"), (40, 64, 2, 0, "forest"), (3, 64, 3, 5, "tree"), (2, 1024, 32, 0, "chain"),
                                                      (3, 1024, 32, 7, "tree"), (2, 1000, 32, 1, "star"), (300, 20, 1, 2, "forest"), (5, 300, 11, 0, "star")])
def test_plan_matches_climbing(binding, B, n_hi, words, window, kind):
    rng = np.random.default_rng(B + n_hi)
    ns = [n_hi] + [int(rng.integers(0, n_hi + 1)) for _ in range(B - 1)]
    parent = sum([_tree.random_parents(rng, n, kind) for n in ns], [])
    cu = np.concatenate(([0], np.cumsum(ns))).tolist()
    kv = [n + int(rng.integers(0, 9000)) for n in ns]
    T = cu[-1] + 5
    _check_plan(binding, parent + [3] * 5, cu, kv, T, words, window, ld=words + B % 3)


def test_plan_refusals_are_per_request(binding):
    """Parents that are not before their row, trees with too many rows, lengths and offsets that make no sense."""
    rng = np.random.default_rng(3)
    ns = [5, 40, 0, 6, 33, 7]
    parent = sum([_tree.random_parents(rng, n) for n in ns], [])
    cu = np.concatenate(([0], np.cumsum(ns))).tolist()
    kv = [9, 50, 0, 5, 40, 100]                          # the fourth: fewer keys than rows
    T = cu[-1] + 2
    parent += [0, 0]
    _check_plan(binding, parent, cu, kv, T, 1)           # the second and fifth do not fit one word
    parent[2], parent[cu[5] + 3], parent[cu[5] + 4], parent[cu[1]] = 2, 2 ** 31 - 1, -2, -2 ** 31
    _check_plan(binding, parent, cu, kv, T, 2)
    for bad in ([0, 5, 3, 45, 51, 84, 91], [-1, 5, 45, 45, 51, 84, 91], [0, 5, 45, 45, 51, 84, T + 1], [0, 5, 45, 45, 51, 84, -7], [0, 5, 45, 45, 51, 84, 46]):
        _check_plan(binding, parent, bad, kv, T, 2)
    big = _tree.random_parents(rng, 1025)
    _check_plan(binding, big, [0, 1025], [2000], 1025, 32)


def test_plan_of_nothing(binding):
    got = binding.tree_plan(i32([]), i32([0]), i32([]), words=1)
    assert got["mask"].shape == (0, 1)
    got = binding.tree_plan(i32([4, 4]), i32([0]), i32([]), words=2)
    assert got["mask"].tolist() == [[0, 0]] * 2 and got["positions"].tolist() == [-1, -1]


# ---- rotate ---------------------------------------------------------------------------------------------------------
def _check_rotate(binding, T, Hq, Hkv, D, rot, dtype, axes=1, neighbours=False, norm=True, page=16, layout="nhd", w_dtype=F32, factor=1.0, far=5000, seed=0, in_place=False, shift=0,
                  bad_axis=False):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    P = -(-T // page) + 2
    caches = [mk(P, page, Hkv, D).to(dtype).cuda() for _ in range(2)]
    if layout == "hnd":
        caches = [c.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for c in caches]
    elif layout == "joined":
        pool = torch.stack(caches, 1).contiguous()
        caches = [pool[:, 0], pool[:, 1]]
    fused = mk(T, Hq + 2 * Hkv, D + shift).to(dtype).cuda()[..., shift:]
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    slot = torch.randperm(P * page, generator=g)[:T].to(torch.int64)
    slot[::5] = -1
    if T > 3:
        slot[1], slot[3] = 2 ** 40, P * page
    pos = torch.randint(-3, far, (axes, T), generator=g, dtype=torch.int64).to(torch.int32)
    half = rot // 2
    inv_freq = (1e4 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()
    axis_of = [i % axes for i in range(half)] if axes > 1 else None
    if bad_axis:
        axis_of = [(-1, axes, 0)[i % 3] for i in range(half)]
    weights = [(1 + 0.3 * mk(D)).to(w_dtype) for _ in range(2)] if norm else [None, None]
    eps = 1e-5 if norm else None
    want_k, want_v = (c.double().cpu() for c in caches)
    tol_k = torch.zeros_like(want_k)
    args = (eps, pos.tolist(), inv_freq, axis_of, neighbours, factor)
    ref_q, tol_q = _tree.rotate_reference(q, weights[0], *args)
    ref_k, bound_k = _tree.rotate_reference(k, weights[1], *args)
    vd = v.double().cpu()
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < P * page:
            want_k[s // page, s % page], tol_k[s // page, s % page], want_v[s // page, s % page] = ref_k[t], bound_k[t], vd[t]
    cw = [None if w is None else w.cuda() for w in weights]
    out = binding.rotate_append(q, k, v, pos.cuda() if axes > 1 or seed % 2 else pos[0].cuda(), inv_freq.cuda(), caches[0], caches[1], slot.cuda(), q_weight=cw[0], k_weight=cw[1], eps=eps,
                                axis_of=None if axis_of is None else i32(axis_of), neighbours=neighbours, factor=factor, q_out=q if in_place else None)
    err = (out.double().cpu() - ref_q).abs()
    assert (err <= tol_q).all(), ((err / tol_q).max(), T, D)
    err = (caches[0].double().cpu() - want_k).abs()
    assert (err <= tol_k).all()
    assert torch.equal(caches[1].double().cpu(), want_v)


ROTATE = [
    # T, Hq, Hkv, D, rot, dtype, further arguments
    (1, 16, 8, 128, 128, BF16, {}), (5, 64, 8, 128, 128, BF16, dict(layout="hnd")), (1300, 8, 2, 128, 128, BF16, {}), (3000, 4, 1, 64, 64, F16, dict(page=64)),
    (77, 7, 3, 128, 64, F16, dict(layout="joined")), (40, 5, 2, 96, 96, BF16, dict(page=7)), (33, 6, 2, 80, 40, BF16, dict(page=24)), (33, 6, 2, 80, 80, F32, {}),
    (20, 4, 4, 256, 256, BF16, {}), (20, 4, 4, 256, 128, F32, {}), (20, 4, 2, 128, 128, F32, dict(neighbours=True)), (50, 9, 2, 64, 64, BF16, dict(neighbours=True)),
    (50, 9, 2, 96, 48, F16, dict(neighbours=True)), (31, 3, 1, 33, 10, BF16, {}), (31, 3, 1, 33, 32, F32, dict(neighbours=True)), (9, 2, 2, 8, 8, F16, {}), (9, 2, 2, 8, 4, BF16, {}),
    (12, 4, 2, 24, 8, BF16, {}), (12, 4, 2, 40, 24, F32, {}), (64, 8, 2, 128, 128, BF16, dict(axes=3)), (64, 8, 2, 128, 128, BF16, dict(axes=2, neighbours=True)),
    (64, 8, 2, 128, 64, F32, dict(axes=4)), (30, 4, 2, 128, 128, BF16, dict(bad_axis=True, axes=2)), (64, 8, 2, 128, 128, F16, dict(norm=False)),
    (64, 8, 2, 64, 32, BF16, dict(norm=False, factor=0.7)), (30, 4, 2, 128, 128, BF16, dict(w_dtype=BF16)), (30, 4, 2, 128, 128, F32, dict(w_dtype=F16)), (30, 4, 2, 64, 0, BF16, {}),
    (30, 4, 2, 64, 64, BF16, dict(far=2 ** 31 - 1)), (30, 4, 2, 64, 64, F32, dict(far=2 ** 31 - 1, axes=3)), (30, 4, 2, 64, 64, BF16, dict(in_place=True)),
    (30, 4, 2, 33, 32, F16, dict(in_place=True)), (30, 4, 2, 64, 64, BF16, dict(shift=1)), (30, 4, 2, 64, 64, BF16, dict(shift=4)), (30, 4, 2, 64, 64, F32, dict(shift=2)),
    (30, 4, 2, 128, 128, F16, dict(shift=2, neighbours=True)), (16, 4, 0, 64, 64, BF16, {}), (16, 0, 3, 64, 64, BF16, {}), (0, 4, 2, 64, 64, BF16, {}),
]


@pytest.mark.parametrize("case", ROTATE, ids=[str(i) for i in range(len(ROTATE))])
def test_rotate_matches_definition(binding, case):
    T, Hq, Hkv, D, rot, dtype, more = case
    _check_rotate(binding, T, Hq, Hkv, D, rot, dtype, seed=T + D + rot, **more)


@pytest.mark.parametrize("seed", range(12))
def test_rotate_random_shapes(binding, seed):
    rng = np.random.default_rng(seed)
    pick = lambda *v: v[int(rng.integers(len(v)))]  # noqa: E731
    D = pick(16, 48, 64, 72, 128, 160, 192, 256, int(rng.integers(1, 257)))
    rot = pick(D // 2 * 2, D // 4 * 2, int(rng.integers(0, D // 2 + 1)) * 2)
    Hq, Hkv = pick(1, 3, 8, 17), pick(1, 2, 5)
    _check_rotate(binding, int(rng.integers(1, 400)), Hq, Hkv, D, rot, pick(BF16, F16, F32), axes=pick(1, 1, 3), neighbours=bool(rng.integers(2)), norm=bool(rng.integers(3)),
                  page=pick(1, 16, 24), layout=pick("nhd", "hnd", "joined"), w_dtype=pick(F32, BF16), far=pick(100, 10 ** 6), seed=100 + seed, shift=pick(0, 0, 1, 4))


@pytest.mark.parametrize("D,rot", [(128, 64), (33, 10)])
def test_rotate_infinities_stay_where_they_are(binding, D, rot):
    """Elements behind the turned ones pass (no norm); rows whose slot names no place leave the caches alone, whatever they hold."""
    T, H = 6, 2
    q = torch.zeros(T, H, D, dtype=BF16, device="cuda")
    q[0, 0, rot], q[1, 1, D - 1], q[2, 0, rot + 3] = INF, -INF, NAN
    k = torch.full((T, H, D), NAN, dtype=BF16, device="cuda")
    kc, vc = (torch.ones(3, 4, H, D, dtype=BF16, device="cuda") for _ in range(2))
    out = binding.rotate_append(q, k, k, i32(list(range(T))), torch.ones(rot // 2, device="cuda"), kc, vc, torch.full((T,), -1, dtype=torch.int64, device="cuda"))
    assert torch.equal(out.isnan(), q.isnan()) and torch.equal(out.nan_to_num(5), q.nan_to_num(5))
    assert (kc == 1).all() and (vc == 1).all()


def test_rotate_beyond_32_bit_offsets(binding):
    P, page, H, D = 140_000, 16, 8, 128
    kc, vc = (torch.empty(P, page, H, D, dtype=BF16, device="cuda") for _ in range(2))
    assert kc.numel() > 2 ** 31
    T = 20
    qkv = torch.randn(T, 3 * H, D, dtype=BF16, device="cuda")
    slot = torch.tensor([(P - 1 - t) * page + t % page for t in range(T)], device="cuda")
    pos, freq = i32(list(range(T))), torch.rand(64, device="cuda")
    binding.rotate_append(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], pos, freq, kc, vc, slot)
    small, small_v = (torch.empty(2, page, H, D, dtype=BF16, device="cuda") for _ in range(2))
    binding.rotate_append(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], pos, freq, small, small_v, torch.arange(T, device="cuda"))
    for t in range(T):
        assert torch.equal(kc[P - 1 - t, t % page], small[t // page, t % page]) and torch.equal(vc[P - 1 - t, t % page], qkv[t, 2 * H:])


# ---- attention ------------------------------------------------------------------------------------------------------
def _masks(rng, lens, kind, words):
    """(mask [T, words] tensor, positions list) of requests with (rows, keys in all)."""
    mask, pos = [np.zeros((0, words), np.int32)], []
    for n, kv in lens:
        if n == 0:
            continue
        if kind in ("tree", "chain", "star", "forest"):
            p = _tree.random_parents(rng, n, kind)
            m, q, _ = _tree.plan_reference(p, [0, n], [max(kv, n)], n, words)
            pos += [x + kv - max(kv, n) for x in q]
        elif kind == "random":                             # any bits, later rows too, some rows without any
            seen = rng.random((n, n)) < 0.4
            seen[rng.random(n) < 0.2] = False
            m = _tree.pack_bits(seen, words)
            pos += [kv - n + int(rng.integers(-2, n + 3)) for _ in range(n)]
        else:
            m = np.zeros((n, words), np.int32)
            pos += [kv - n] * n
        mask.append(m)
    return np.concatenate(mask), pos


def _attend(binding, lens, Hq, Hkv, D, page, dtype, window=0, layout="nhd", kind="tree", seed=0, generic=False, spare_words=0, scale=None, q_factor=1.0):
    rng = np.random.default_rng(seed)
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", seed, layout, width_extra=seed % 3)
    words = max(1, (max(n for n, _ in lens) + 31) // 32) + spare_words
    mask, pos = _masks(rng, lens, kind, words)
    mask = torch.tensor(np.concatenate([mask, np.full((3, words), -1, np.int32)]), device="cuda")
    pos = i32(pos + [5] * 3)
    q = (torch.randn(T + 3, Hq, D, generator=g) * q_factor).to(dtype).cuda()
    out, lse, status = torch.full_like(q, 7.0), torch.full((T + 3, Hq), 7.0, device="cuda"), i32([0] * len(lens))
    got, got_lse = binding.tree_attention(q, kc, vc, table, i32(cu), i32(kv), mask, positions=pos, scale=scale, window=window, out=out, lse=lse, status=status, generic=generic)
    assert got is out and got_lse is lse
    ref = _tree.attention_reference(q, kc, vc, table, cu, kv, mask, 1.0 / math.sqrt(D) if scale is None else scale, window, pos.tolist())
    return out, lse, status, ref


def _compare(out, lse, ref):
    want, want_lse, tol, tol_lse, written = ref
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (o[~written] == 7.0).all() and (l[~written] == 7.0).all()          # rows of no request are left as they were
    empty = np.isneginf(want_lse) & written[:, None]
    assert np.isneginf(l[empty]).all() and (o[empty] == 0).all()
    live = written[:, None] & ~empty
    err, bound = np.abs(o - want)[live], tol[live]
    assert np.isfinite(o[live]).all()
    assert (err <= bound).all(), (err / bound).max()
    err, bound = np.abs(l - want_lse)[live], tol_lse[live]
    assert (err <= bound).all(), (err / bound).max()


SHAPES = [
    # lens [(rows, keys in all)], Hq, Hkv, D, page, dtype, window, layout, mask
    ("one_row", [(1, 1)], 1, 1, 64, 16, BF16, 0, "nhd", "tree"),
    ("rows_and_nothing_before", [(9, 9), (40, 40), (1, 1)], 8, 2, 128, 16, BF16, 0, "nhd", "tree"),
    ("small_trees", [(9, 9), (9, 133), (9, 137), (9, 1027)], 16, 8, 128, 16, BF16, 0, "nhd", "tree"),
    ("idle_requests", [(0, 50), (3, 70), (0, 0), (6, 6), (0, 9)], 8, 1, 64, 32, F16, 0, "hnd", "tree"),
    ("no_bits", [(9, 9), (9, 140), (33, 33)], 4, 2, 128, 16, BF16, 0, "nhd", "none"),
    ("random_bits", [(9, 200), (70, 333), (33, 33), (130, 300)], 4, 2, 128, 16, BF16, 0, "nhd", "random"),
    ("random_bits_no_groups", [(200, 420), (31, 64)], 2, 2, 64, 64, F16, 0, "nhd", "random"),
    ("wide", [(64, 700), (63, 900)], 8, 2, 128, 64, BF16, 0, "nhd", "star"),
    ("forest", [(64, 130), (40, 300)], 8, 2, 128, 16, BF16, 0, "nhd", "forest"),
    ("many_rows", [(300, 700), (257, 257)], 4, 1, 128, 64, BF16, 0, "nhd", "tree"),
    ("all_rows", [(1024, 1100)], 2, 1, 64, 64, BF16, 0, "nhd", "tree"),
    ("page_of_8", [(14, 77), (22, 260)], 4, 2, 64, 8, BF16, 0, "nhd", "tree"),
    ("page_of_256", [(25, 700), (12, 256)], 8, 2, 64, 256, BF16, 0, "nhd", "tree"),
    ("page_of_24", [(15, 100), (1, 24)], 6, 2, 128, 24, BF16, 0, "nhd", "tree"),
    ("width_80", [(15, 200), (40, 200)], 6, 2, 80, 16, BF16, 0, "joined", "tree"),
    ("width_33", [(14, 60)], 4, 2, 33, 16, BF16, 0, "nhd", "random"),
    ("width_256", [(13, 90), (20, 50)], 4, 2, 256, 16, BF16, 0, "nhd", "tree"),
    ("groups_of_7", [(29, 150), (50, 150)], 14, 2, 64, 16, BF16, 0, "hnd", "tree"),
    ("group_of_16", [(29, 400), (70, 400)], 16, 1, 128, 32, BF16, 0, "nhd", "tree"),
    ("group_of_40", [(12, 300)], 40, 1, 64, 16, BF16, 0, "nhd", "tree"),
    ("group_of_136", [(5, 70)], 136, 1, 64, 16, BF16, 0, "nhd", "tree"),
    ("window_1", [(15, 200), (1, 1), (40, 100)], 4, 2, 64, 16, BF16, 1, "nhd", "tree"),
    ("window_below_the_depth", [(40, 300), (40, 40)], 4, 2, 64, 16, BF16, 9, "nhd", "chain"),
    ("window_in_tile", [(15, 300), (200, 450)], 4, 2, 128, 16, BF16, 37, "nhd", "tree"),
    ("window_over_tiles", [(15, 900), (150, 700), (3, 100)], 8, 2, 128, 64, BF16, 300, "hnd", "tree"),
    ("window_random", [(35, 900), (70, 500)], 8, 2, 128, 64, BF16, 130, "nhd", "random"),
    ("window_past_all", [(15, 300), (1, 1)], 4, 2, 64, 16, BF16, 2 ** 31 - 1, "nhd", "tree"),
    ("many_requests", [(1 + i % 19, 20 + (i * 37) % 300) for i in range(90)], 4, 2, 64, 16, BF16, 0, "nhd", "tree"),
    ("long_context", [(45, 9001)], 4, 1, 128, 64, BF16, 0, "nhd", "tree"),
]


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("case", SHAPES, ids=[c[0] for c in SHAPES])
def test_attention_matches_reference(binding, case, generic):
    name, lens, Hq, Hkv, D, page, dtype, window, layout, kind = case
    out, lse, status, ref = _attend(binding, lens, Hq, Hkv, D, page, dtype, window, layout, kind, seed=len(name), generic=generic, spare_words=len(name) % 2)
    _compare(out, lse, ref)
    assert (status == 0).all()


@pytest.mark.parametrize("seed", range(16))
def test_attention_random_shapes(binding, seed):
    rng = np.random.default_rng(500 + seed)
    pick = lambda *v: v[int(rng.integers(len(v)))]  # noqa: E731
    Hkv, G, D, page = pick(1, 2, 3), pick(1, 2, 3, 4, 5, 8, 12, 16), 8 * int(rng.integers(1, 17)), pick(8, 16, 32, 64, 128, 192)
    lens = []
    for _ in range(int(rng.integers(1, 7))):
        n = pick(0, 1, int(rng.integers(1, 20)), int(rng.integers(1, 90)), int(rng.integers(1, 400 // G + 2)))
        lens.append((n, n + pick(0, 1, int(rng.integers(0, 130)), int(rng.integers(0, 700)))))
    out, lse, status, ref = _attend(binding, lens, Hkv * G, Hkv, D, page, pick(BF16, F16), pick(0, 0, int(rng.integers(1, 300))), pick("nhd", "hnd", "joined"),
                                    pick("tree", "random", "chain", "forest"), seed=seed, spare_words=seed % 3)
    _compare(out, lse, ref)
    assert (status == 0).all()


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 64)])
def test_a_chain_is_the_chunk_attention(binding, D, page, window):
    """Masks of chains: the same as chunk_attention but for the order of sums (a rounding of the weights, one of the result: each
    is within its own bound of the exact values)."""
    lens = [(5, 300), (40, 700), (130, 200)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, 2, D, BF16, "cuda", 5)
    q = torch.randn(T, 8, D, generator=g).to(BF16).cuda()
    parent = sum([list(range(-1, n - 1)) for n, _ in lens], [])
    plan = binding.tree_plan(i32(parent), i32(cu), i32(kv), words=5, window=window)
    a, la = binding.tree_attention(q, kc, vc, table, i32(cu), i32(kv), plan["mask"], positions=plan["positions"], window=window)
    b, lb = binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), window=window)
    ref = _paged.attention_reference(q, kc, vc, table, cu, kv, 1 / math.sqrt(D), window)
    for o, l in ((a, la), (b, lb)):
        assert (np.abs(o.double().cpu().numpy() - ref[0]) <= ref[2]).all() and (np.abs(l.double().cpu().numpy() - ref[1]) <= ref[3]).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("n", [12, 70])
def test_attention_keys_a_row_does_not_see_do_not_reach_it(binding, n, generic):
    """NaN and infinities in keys and values of the chunk: rows without their bit are what they are without them."""
    kc, vc, table, cu, kv, T, g = build_cache([(n, n + 150)], 16, 2, 128, BF16, "cuda", 3)
    q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
    rng = np.random.default_rng(n)
    parent = _tree.random_parents(rng, n)
    mask, _, _ = _tree.plan_reference(parent, cu, kv, T, 3)
    mask = torch.tensor(mask, device="cuda")
    spoilt_k, spoilt_v = 1, n // 2                        # rows of the chunk
    for r, cache, head, e, x in ((spoilt_k, kc, 1, 5, NAN), (spoilt_v, vc, 0, 77, INF)):
        j = 150 + r
        cache[int(table[0, j // 16]), j % 16, head, e] = x
    out, lse = binding.tree_attention(q, kc, vc, table, i32(cu), i32(kv), mask, generic=generic)
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    want, want_lse, tol, tol_lse, _ = _tree.attention_reference(q, kc, vc, table, cu, kv, mask, 1 / math.sqrt(128))
    for i in range(n):
        way = _tree.climb(parent, i)
        keep = np.ones((8, 128), bool)
        if spoilt_v in way:
            assert np.isposinf(o[i, :4, 77]).all()
            keep[:4, 77] = False
        if spoilt_k in way:
            assert np.isnan(o[i, 4:]).all() and np.isnan(l[i, 4:]).all()
            keep[4:] = False
        assert (np.abs(o[i] - want[i])[keep] <= tol[i][keep]).all(), i
        rows = keep.all(1) | (np.arange(8) < 4)
        assert (np.abs(l[i] - want_lse[i])[rows] <= tol_lse[i][rows]).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_refuses_requests(binding, generic):
    """Fewer keys than rows, more rows than bits, lengths and offsets that make no sense, pages that are gone."""
    lens = [(5, 100), (40, 90), (6, 300), (33, 60), (4, 20)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 64, BF16, "cuda", 11)
    rng = np.random.default_rng(1)
    q = torch.randn(T, 4, 64, generator=g).to(BF16).cuda()
    mask, pos = _masks(rng, lens, "tree", 2)
    mask = torch.tensor(mask, device="cuda")
    table[2, 1] = kc.shape[0]

    def call(cu_, kv_, m):
        out, lse, status = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda"), i32([0] * 5)
        binding.tree_attention(q, kc, vc, table, i32(cu_), i32(kv_), m, out=out, lse=lse, status=status, generic=generic)
        _compare(out, lse, _tree.attention_reference(q, kc, vc, table, cu_, kv_, m, 1 / 8))
        return status.tolist()
    assert call(cu, kv, mask) == [0, 0, BAD_PAGE, 0, 0]
    assert call(cu, kv, mask[:, :1]) == [0, BAD_LEN, BAD_PAGE, BAD_LEN, 0]     # (a mask with rows wider than what is read)
    assert call(cu, [4, 39] + kv[2:], mask) == [BAD_LEN, BAD_LEN, BAD_PAGE, 0, 0]
    assert call(cu, [-1, 2 ** 31 - 1] + kv[2:], mask) == [BAD_LEN, BAD_LEN, BAD_PAGE, 0, 0]
    assert call([0, 5, 3] + cu[3:], kv, mask)[1] == BAD_LEN
    assert call(cu[:5] + [T + 1], kv, mask) == [0, 0, BAD_PAGE, 0, BAD_LEN]


def test_attention_pages_behind_the_window_may_be_gone(binding):
    lens = [(20, 900), (7, 500)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 64, BF16, "cuda", 17)
    q = torch.randn(T, 4, 64, generator=g).to(BF16).cuda()
    rng = np.random.default_rng(2)
    mask, pos = _masks(rng, lens, "tree", 1)
    mask = torch.tensor(mask, device="cuda")
    for b, (n, total) in enumerate(lens):
        first = total - n - 100 + 1
        table[b, :first // 16] = -5
    for generic in (False, True):
        out, lse, status = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda"), i32([0, 0])
        binding.tree_attention(q, kc, vc, table, i32(cu), i32(kv), mask, positions=i32(pos), window=100, out=out, lse=lse, status=status, generic=generic)
        _compare(out, lse, _tree.attention_reference(q, kc, vc, table, cu, kv, mask, 1 / 8, 100, pos))
        assert status.tolist() == [0, 0]


@pytest.mark.parametrize("lens,stops", [([(9, 30009), (0, 9), (40, 700)], (0, 2)), ([(63, 9000)] * 3, (0, 4))])
def test_attention_waits_that_run_out_are_reported(binding, lens, stops):
    """CTAs that stop loading keys: the waits run out, the kernel ends by itself, says TIMEOUT and leaves NaN; the next call is as before."""
    kc, vc, table, cu, kv, T, g = build_cache(lens, 64, 1, 128, BF16, "cuda", 80)
    q = torch.randn(T + 2, 8, 128, generator=g).to(BF16).cuda()
    mask = torch.tensor(np.concatenate([_masks(np.random.default_rng(0), lens, "tree", 2)[0], np.zeros((2, 2), np.int32)]), device="cuda")
    args = (q, kc, vc, table, i32(cu), i32(kv), mask)

    def call(**k):
        out, lse, status = torch.full_like(q, 7.0), torch.full((T + 2, 8), 7.0, device="cuda"), i32([0] * len(lens))
        binding.tree_attention(*args, out=out, lse=lse, status=status, **k)
        torch.cuda.synchronize()
        assert (out[T:] == 7).all()
        return out, lse, int(status[0])
    want, want_lse, status = call()
    assert status == 0
    for blocks in stops:
        out, lse, status = call(stop_after=blocks)
        assert status == binding.REQ_TIMEOUT and out[:T].isnan().all() and lse[:T].isnan().all()
        out, lse, status = call()
        assert status == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_attention_strides_and_same_bits(binding):
    """q inside a projection's output, a mask with wider rows, a caller's workspace, other streams: the same bits."""
    lens = [(15, 2000), (45, 70), (1, 900)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 13)
    fused = torch.randn(T, 12 * 128, generator=g).to(BF16).cuda()
    q = fused[:, :1024].view(T, 8, 128)
    wide = torch.full((T, 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :2] = torch.tensor(_masks(np.random.default_rng(4), lens, "tree", 2)[0], device="cuda")
    cu_t, kv_t = i32(cu), i32(kv)
    first, lse = binding.tree_attention(q.contiguous(), kc, vc, table, cu_t, kv_t, wide[:, :2].contiguous())
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [binding.tree_attention(q, kc, vc, table, cu_t, kv_t, wide[:, :2]), binding.tree_attention(q, kc, vc, table, cu_t, kv_t, wide[:, :2], workspace=room)]
    for _ in range(3):
        got += [binding.tree_attention(q, kc, vc, table, cu_t, kv_t, wide[:, :2], stream=s) for s in streams]
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, first) and torch.equal(l, lse)


# ---- log probabilities ----------------------------------------------------------------------------------------------
def _check_logprobs(binding, x, tokens=None, temperature=None, top=0):
    """x: logits on the GPU with finite or -inf entries, every row with a finite one."""
    R, V = x.shape
    status = i32([0] * R)
    got = binding.token_logprobs(x, tokens, temperature=temperature, top=top, status=status)
    assert (status == 0).all()
    logp, lse, entropy, tol_lse, tol_h, tol_p = _tree.logprobs_reference(x, temperature)
    err = (got["lse"].double().cpu() - lse).abs()
    assert (err <= tol_lse).all(), (err / tol_lse).max()
    err = (got["entropy"].double().cpu() - entropy).abs()
    assert (err <= tol_h).all(), (err / tol_h).max()

    def near(a, lp, rows):
        a = a.double().cpu()
        inf = torch.isneginf(lp)
        assert torch.equal(torch.isneginf(a), inf)
        bound = tol_p[rows] + 6 * 2.0 ** -24 * lp.abs()
        assert ((a - lp).abs()[~inf] <= bound[~inf]).all()
    if tokens is not None:
        t = tokens.cpu().reshape(R, -1).long()
        lp = torch.where((t >= 0) & (t < V), logp.gather(1, t.clamp(0, V - 1)), torch.full(t.shape, -INF, dtype=torch.float64))
        assert got["logprob"].shape == tokens.shape
        near(got["logprob"].reshape(R, -1).reshape(-1), lp.reshape(-1), torch.arange(R).repeat_interleave(t.shape[1]))
    if top:
        ids = _tree.top_reference(x, top)
        assert torch.equal(got["top_id"].long().cpu(), ids)
        near(got["top_logprob"].reshape(-1), logp.gather(1, ids).reshape(-1), torch.arange(R).repeat_interleave(top))
    return got


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 7), (4, 33), (9, 255), (6, 1000), (1, 4099), (300, 1111), (900, 1111), (40, 32000), (150, 31000), (3, 151936), (1, 256000), (1, 300001)])
def test_logprobs_match_definition(binding, R, V, dtype):
    g = torch.Generator().manual_seed(R + V)
    x = (torch.randn(R, V, generator=g) * 3).to(dtype).cuda()
    tokens = torch.randint(0, V, (R, 3), generator=g, dtype=torch.int32).cuda()
    tokens[0, 1] = -1
    temperature = (torch.rand(R, generator=g) * 2 + 0.05).cuda()
    _check_logprobs(binding, x, tokens, temperature, min(V, 20))
    _check_logprobs(binding, x, tokens[:, 0].contiguous(), None, min(V, 32))
    _check_logprobs(binding, x, top=1)
    _check_logprobs(binding, x)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("off,ld", [(0, 1001), (1, 1003), (3, 1008), (7, 1040)])
@pytest.mark.parametrize("R", [12, 170, 760])
def test_logprobs_of_rows_of_any_alignment(binding, R, off, ld, dtype):
    g = torch.Generator().manual_seed(off + ld)
    buf = torch.full((R * ld + 16,), NAN).to(dtype)
    x = buf.cuda()[off:off + R * ld].view(R, ld)[:, :1000]
    x.copy_((torch.randn(R, 1000, generator=g) * 3).to(dtype))
    _check_logprobs(binding, x, torch.randint(0, 1000, (R,), generator=g, dtype=torch.int32).cuda(), None, 9)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("kind", ["flat", "masked", "lowest", "half_masked", "ascending", "descending", "one_spike", "ties", "two_values", "huge", "all_lowest"])
@pytest.mark.parametrize("R,V", [(4, 700), (4, 40003), (170, 5003), (760, 700), (760, 5003)])
def test_logprobs_of_odd_rows(binding, R, V, kind, dtype):
    """Rows with many equal entries, masked vocabularies, sorted rows, a spike, values next to the type's end."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(R, V, generator=g).to(dtype)
    low = torch.finfo(dtype).min
    if kind == "flat":
        x.zero_()
        x[1] = -0.0
        x[1, ::2] = 0.0
    elif kind in ("masked", "lowest"):
        y = x[:, 100:107].clone()
        x.fill_(-INF if kind == "masked" else low)
        x[:, 100:107] = y
    elif kind == "half_masked":
        x[torch.rand(R, V, generator=g) < 0.5] = -INF
    elif kind in ("ascending", "descending"):
        x = torch.linspace(-4, 4, V).to(dtype).repeat(R, 1)
        if kind == "descending":
            x = x.flip(1)
    elif kind == "one_spike":
        x[:, V // 3] = 90
        x[2, V - 1] = 91
    elif kind == "ties":
        x = torch.randint(0, 5, (R, V), generator=g).to(dtype)
    elif kind == "two_values":
        x = torch.where(torch.rand(R, V, generator=g) < 0.01, 1.0, 0.0).to(dtype)
    elif kind == "huge":
        x = x * (torch.finfo(dtype).max / 64)
        x[torch.isinf(x)] = 0
    elif kind == "all_lowest":
        x.fill_(low)
    if kind in ("huge", "all_lowest") and dtype != F16:
        # the largest l is next to float32's end, where nothing but the likeliest entries and its own rounding is left
        got = binding.token_logprobs(x.cuda(), top=20)
        assert torch.equal(got["top_id"].long().cpu(), _tree.top_reference(x, 20))
        want = torch.logsumexp(x.double(), 1)
        assert ((got["lse"].double().cpu() - want).abs() <= want.abs() * 2.0 ** -23).all()
        if kind == "all_lowest":
            assert (got["entropy"].double().cpu() - math.log(V)).abs().max() <= 2.0 ** -12 and (got["top_logprob"].double().cpu() + math.log(V)).abs().max() <= 2.0 ** -12
        return
    for top in (1, 20, 32):
        _check_logprobs(binding, x.cuda(), torch.randint(0, V, (R, 2), generator=g, dtype=torch.int32).cuda(), None, top)


@pytest.mark.parametrize("V", [50, 9001])
@pytest.mark.parametrize("times", [1, 20, 80])
def test_logprobs_of_rows_that_have_none(binding, times, V):
    """NaN, +inf, nothing but -inf, temperatures that make no sense, tokens outside: said in the status, the others as alone."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn(10, V, generator=g).cuda()
    temp = torch.ones(10, device="cuda")
    x[1, V - 1], x[2, 7], x[3] = NAN, INF, -INF
    x[8] = NAN
    temp[4], temp[5], temp[6], temp[7] = 0, -1, NAN, INF
    tokens = torch.zeros(10, 3, dtype=torch.int32, device="cuda")
    tokens[0] = i32([V, -1, 3])
    tokens[1, 0], tokens[9] = -2, i32([2 ** 31 - 1, -2 ** 31, V - 1])
    status = i32([0] * 10 * times)
    got = binding.token_logprobs(x.repeat(times, 1), tokens.repeat(times, 1), temperature=temp.repeat(times), top=4, status=status)
    for k in got:   # (the sums of equal rows may be cut at different places)
        a, b = got[k], got[k][:10].repeat([times] + [1] * (got[k].dim() - 1))
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf()) and (a.nan_to_num(7, 8, 9) - b.nan_to_num(7, 8, 9)).abs().max() < 1e-4
    assert torch.equal(status, status[:10].repeat(times))
    got, status = {k: v[:10] for k, v in got.items()}, status[:10]
    NONFINITE, BAD_TOKEN, BAD_PARAM = binding.REQ_NONFINITE, binding.REQ_BAD_TOKEN, binding.REQ_BAD_PARAM
    assert status.tolist() == [BAD_TOKEN, NONFINITE | BAD_TOKEN, NONFINITE, NONFINITE] + [BAD_PARAM] * 4 + [NONFINITE, BAD_TOKEN]
    for r in range(1, 9):
        assert all(got[k][r].isnan().all() for k in ("lse", "entropy", "logprob", "top_logprob")) and (got["top_id"][r] == -1).all()
    alone = binding.token_logprobs(x[[0, 9]].contiguous(), tokens[[0, 9]].contiguous(), top=4)
    ref = torch.log_softmax(x[[0, 9]].double(), 1)
    assert torch.isneginf(got["logprob"][0, :2]).all() and torch.isneginf(got["logprob"][9, :2]).all()
    assert (got["logprob"][[0, 9], 2].double() - torch.stack((ref[0, 3], ref[1, V - 1]))).abs().max() < 1e-4
    for k in ("top_id",):
        assert torch.equal(alone[k], got[k][[0, 9]])
    tiny = binding.token_logprobs(x[:1], temperature=torch.full((1,), 1e-39, device="cuda"), status=(s := i32([0])))
    assert tiny["lse"].isnan().all() and s.tolist() == [NONFINITE]


def test_logprobs_of_nothing_and_many_tokens(binding):
    x = torch.randn(3, 500, device="cuda")
    got = binding.token_logprobs(x[:0], torch.empty(0, 2, dtype=torch.int32, device="cuda"), top=3)
    assert got["logprob"].shape == (0, 2) and got["top_id"].shape == (0, 3)
    _check_logprobs(binding, x, torch.arange(500, dtype=torch.int32, device="cuda").repeat(3, 1), None, 5)   # more tokens than a block has threads
    one = x[:1].expand(4, 500)
    with pytest.raises(binding.SpecSteerError) as e:                                                          # rows that share memory: a stride below V
        binding.token_logprobs(one)
    assert e.value.code == binding.ERR_INVALID_ARG


def test_logprobs_beyond_32_bit_offsets(binding):
    """Rows more than 2^31 elements apart."""
    ld, V = 2 ** 31 + 24, 5000
    buf = torch.empty(ld + V, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(1)
    rows = (torch.randn(2, V, generator=g) * 3).to(BF16).cuda()
    buf[:V], buf[ld:] = rows[0], rows[1]
    x = buf.as_strided((2, V), (ld, 1))
    got, want = binding.token_logprobs(x, top=7), binding.token_logprobs(rows, top=7)
    for k in got:
        assert torch.equal(got[k], want[k]), k


def test_logprobs_many_rows_same_bits(binding):
    """More rows than warps and fewer; the same bits again, on other streams at once, and in a captured graph."""
    g = torch.Generator().manual_seed(9)
    for R, V in ((5000, 600), (17, 70001)):
        x = (torch.randn(R, V, generator=g) * 3).to(BF16).cuda()
        tok = torch.randint(0, V, (R,), generator=g, dtype=torch.int32).cuda()
        first = _check_logprobs(binding, x, tok, None, 8)
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        got = [binding.token_logprobs(x, tok, top=8, stream=s) for s in streams for _ in range(2)]
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            got.append(binding.token_logprobs(x, tok, top=8))
        graph.replay()
        torch.cuda.synchronize()
        for o in got:
            for k in first:
                assert torch.equal(o[k], first[k]), k


# ---- keep -----------------------------------------------------------------------------------------------------------
def _drafts(rng, ns, hit=0.8, kinds=("tree",), vocabulary=9):
    """Parents, tokens and choices of trees whose choices mostly are a child's token."""
    parent, token, choice = [], [], []
    for b, n in enumerate(ns):
        p = _tree.random_parents(rng, n, kinds[b % len(kinds)])
        t = [int(x) for x in rng.integers(0, vocabulary, n)]
        c = [int(x) for x in rng.integers(0, vocabulary, n)]
        for i in range(n):
            kids = [j for j in range(i + 1, n) if p[j] == i]
            if kids and rng.random() < hit:
                c[i] = t[kids[int(rng.integers(len(kids)))]]
        parent, token, choice = parent + p, token + t, choice + c
    return parent, token, choice


def _check_keep(binding, ns, pasts, page, layers, H, D, dtype, max_out, layout="nhd", seed=0, kinds=("tree",), table_hook=None):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    kv = [n + p for n, p in zip(ns, pasts)]
    need = [-(-x // page) for x in kv]
    P, W = sum(need) + 2, max(need + [1]) + 1
    perm = torch.randperm(P, generator=g).tolist()
    table = np.full((len(ns), W), -3, np.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = perm[at:at + m]
        at += m
    if table_hook:
        table_hook(table, P)
    parent, token, choice = _drafts(rng, ns, kinds=kinds)
    cu = np.concatenate(([0], np.cumsum(ns))).astype(int).tolist()
    T = cu[-1] + 2
    parent, token, choice = parent + [0, 0], token + [1, 1], choice + [1, 1]
    shape = (P, page, H, D) if layers == 0 else (layers, P, page, H, D)
    caches = []
    for _ in range(2):
        c = torch.randn(*shape, generator=g).to(dtype).cuda()
        if layout == "hnd":
            c = c.transpose(-2, -3).contiguous().transpose(-2, -3)
        caches.append(c)
    n_out, path, toks, moves, status = _tree.keep_reference(parent, token, choice, cu, kv, T, max_out, table, page, P)
    want = [c.clone().flatten(-4, -3) for c in caches]
    for src, dst in moves:                                # in order: a later place is never the source of an earlier row
        for w in want:
            w[..., dst, :, :] = w[..., src, :, :]
    st = i32([0] * len(ns))
    got = binding.tree_keep(i32(parent), i32(token), i32(choice), i32(cu), i32(kv), torch.tensor(table, device="cuda"), caches[0], caches[1], max_out=max_out, status=st)
    assert got["n_out"].tolist() == n_out and got["path"].tolist() == path and got["out_tokens"].tolist() == toks
    assert st.tolist() == status
    for c, w in zip(caches, want):
        assert torch.equal(c.flatten(-4, -3), w)
    return n_out, moves


@pytest.mark.parametrize("ns,pasts,page,layers,H,D,dtype,max_out,layout", [
    ([9], [715], 16, 3, 8, 128, BF16, 6, "nhd"), ([1, 0, 1], [0, 0, 5], 16, 2, 1, 64, F16, 3, "nhd"), ([30, 25, 0, 64, 7], [0, 13, 4, 127, 300], 16, 2, 2, 64, BF16, 9, "hnd"),
    ([30] * 9, list(range(9)), 1, 0, 2, 96, F32, 8, "nhd"), ([40, 40], [5, 6], 7, 5, 3, 33, F16, 12, "nhd"), ([20, 33], [3, 60], 24, 1, 1, 5, F32, 4, "hnd"),
    ([200, 17], [3, 64], 64, 2, 2, 128, BF16, 1, "nhd"), ([12] * 70, [31] * 70, 32, 4, 8, 128, BF16, 7, "nhd"), ([60, 60], [1, 2], 16, 1, 300, 256, BF16, 30, "nhd")])
def test_keep_matches_reference(binding, ns, pasts, page, layers, H, D, dtype, max_out, layout):
    _check_keep(binding, ns, pasts, page, layers, H, D, dtype, max_out, layout, seed=len(ns) + D, kinds=("tree", "forest"))


@pytest.mark.parametrize("seed", range(6))
def test_keep_long_paths(binding, seed):
    """Chains and narrow trees, whose paths are long and move a little at every step; the most rows a tree may have."""
    n_out, moves = _check_keep(binding, [300, 1024, 700], [10, 33, 0], 16, 1, 1, 32, BF16, 1024, seed=seed, kinds=("chain", "tree", "forest"))
    assert len(moves) > 0


def test_keep_takes_the_lowest_of_equal_siblings(binding):
    got = binding.tree_keep(i32([-1, 0, 0, 1, 2]), i32([9, 4, 4, 5, 5]), i32([4, 5, 5, 6, 7]), i32([0, 5]), i32([5]), max_out=4)
    assert got["path"].tolist() == [[0, 1, 3, -1]] and got["out_tokens"].tolist() == [[4, 5, 6, -1]] and got["n_out"].tolist() == [3]


def test_keep_negative_choices_are_nobodys_token(binding):
    """Rows without probabilities choose -1, which a padded draft's token of -1 must not confirm."""
    got = binding.tree_keep(i32([-1, 0, 1, -1, 0]), i32([3, -1, -1, 2, 8]), i32([-1, -1, -1, 8, -5]), i32([0, 3, 5]), i32([3, 2]), max_out=4)
    assert got["path"].tolist() == [[0, -1, -1, -1], [0, 1, -1, -1]] and got["out_tokens"].tolist() == [[-1, -1, -1, -1], [8, -5, -1, -1]] and got["n_out"].tolist() == [1, 2]


def test_keep_refuses_requests(binding):
    """Bad pages leave their token where it is; lengths that make no sense keep nothing; odd parents belong to nobody."""
    def hook(table, P):
        table[0, 0], table[1, 2] = P, -1
    _check_keep(binding, [60, 60, 60], [5, 20, 7], 16, 2, 2, 64, BF16, 12, seed=3, table_hook=hook)
    parent, token, choice = i32([-1, 0, 1, -1, 7, 2, -1, 0]), i32([1] * 8), i32([1] * 8)
    table = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    kc, vc = (torch.arange(64 * 8, device="cuda").to(BF16).view(4, 16, 1, 8) for _ in range(2))
    before = kc.clone()
    for cu, kv, want in (([0, 3, 6, 8], [2, 65, 2], [BAD_LEN, BAD_LEN, 0]), ([0, 3, 2, 9], [3, 5, 9], [0, BAD_LEN, BAD_LEN]), ([-1, 3, 6, 8], [9, 3, 2], [BAD_LEN, 0, 0])):
        st = i32([0] * 3)
        got = binding.tree_keep(parent, token, choice, i32(cu), i32(kv), table, kc, vc, max_out=4, status=st)
        assert st.tolist() == want
        for b in range(3):
            if want[b]:
                assert got["n_out"][b] == 0 and got["path"][b].tolist() == [-1] * 4 and got["out_tokens"][b].tolist() == [-1] * 4
        assert torch.equal(kc, before)                    # (their paths begin with their first rows: nothing moves)
    got = binding.tree_keep(parent, token, choice, i32([0, 3, 6, 8]), i32([3, 3, 2]), max_out=4)
    assert got["n_out"].tolist() == [3, 1, 2]             # the second request's rows name parents behind themselves
    with pytest.raises(ValueError):
        binding.tree_keep(parent, token, choice, i32([0, 3, 6, 8]), i32([3, 3, 2]), table.cpu(), kc, vc, max_out=4)


def test_keep_beyond_32_bit_offsets(binding):
    P, page, H, D = 140_000, 16, 8, 128
    kc, vc = (torch.empty(P, page, H, D, dtype=BF16, device="cuda") for _ in range(2))
    pages = [P - 1, P - 5]
    kc[pages], vc[pages] = (torch.randn(2, page, H, D, dtype=BF16, device="cuda") for _ in range(2))
    want = [c[pages].flatten(0, 1).clone() for c in (kc, vc)]
    binding.tree_keep(i32([-1, 0, 0, 2, 0, 3, 5]), i32([0, 1, 2, 3, 4, 5, 6]), i32([2, 0, 3, 5, 0, 6, 8]), i32([0, 7]), i32([20]), i32([pages]), kc, vc, max_out=9)   # path 0 2 3 5 6
    for c, w in zip((kc, vc), want):
        for i, j in enumerate((0, 2, 3, 5, 6)):
            w[13 + i] = w[13 + j].clone()
        assert torch.equal(c[pages].flatten(0, 1), w)


# ---- a run of them together -------------------------------------------------------------------------------------------
def _round_state(B, page, W, P, layers, H, D, seed):
    g = torch.Generator().manual_seed(seed)
    return {"seq_len": i32([0] * B), "held": i32([0] * B), "table": torch.full((B, W), -1, dtype=torch.int32, device="cuda"), "ring": torch.randperm(P, generator=g).to(torch.int32).cuda(),
            "pos": torch.tensor([0, P], device="cuda"), "kc": torch.full((layers, P, page, H, D), NAN, dtype=BF16, device="cuda"),
            "vc": torch.full((layers, P, page, H, D), NAN, dtype=BF16, device="cuda")}


def test_rounds_over_trees(binding):
    """Prompt, then rounds: plan -> tree plan -> rotate and append -> attention -> log probabilities -> keep -> plan with its n_out,
    nothing read back in between.  The rows of the path give what a chain of the same tokens gives, and the cache holds
    the kept tokens' keys and values in order, whatever was drafted beside them."""
    B, Hq, Hkv, D, page, W, P, layers, V = 5, 8, 2, 64, 16, 14, 60, 2, 211
    st = _round_state(B, page, W, P, layers, Hkv, D, 1)
    g = torch.Generator().manual_seed(2)
    rng = np.random.default_rng(3)
    emb = torch.randn(V, (Hq + 2 * Hkv) * D, generator=g).to(BF16).cuda()       # a token's projections, the same in every round
    head = (torch.randn(Hq * D, V, generator=g) / 8).to(BF16).cuda()
    freq = (1e4 ** (-torch.arange(D // 2) / (D // 2))).cuda()
    weights = [torch.rand(D, generator=g).cuda() + 0.5 for _ in range(2)]
    hist = [[int(x) for x in rng.integers(0, V, n)] for n in (3, 17, 30, 1, 9)]  # the tokens in each cache
    advance, new = None, i32([len(h) for h in hist])
    out_tokens = None

    def forward(tokens, plan, positions, mask):
        x = emb[tokens.long().clamp(min=0)].view(-1, Hq + 2 * Hkv, D)
        for layer in range(layers):
            q = binding.rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], positions, freq, st["kc"][layer], st["vc"][layer], plan["slot_map"], q_weight=weights[0],
                                      k_weight=weights[1], eps=1e-6)
            if mask is None:
                o, _ = binding.chunk_attention(q, st["kc"][layer], st["vc"][layer], st["table"], plan["cu_new"], plan["kv_len"], status=plan["status"])
            else:
                o, _ = binding.tree_attention(q, st["kc"][layer], st["vc"][layer], st["table"], plan["cu_new"], plan["kv_len"], mask, status=plan["status"])
        return o.reshape(len(o), -1).nan_to_num(0) @ head

    for step in range(6):
        ns = [len(h) for h in hist] if step == 0 else [1 + int(rng.integers(0, 20)) for _ in range(B)]
        T = sum(ns) + 2
        plan = binding.cache_plan(st["seq_len"], i32(ns) if step else new, st["held"], st["table"], st["ring"], st["pos"], page_size=page, max_tokens=T, advance=advance)
        st.update(seq_len=plan["seq_len"], held=plan["pages_held"], pos=plan["ring_pos"])
        cu = plan["cu_new"].tolist()
        if step == 0:
            tokens = i32(sum(hist, []) + [0, 0])
            logits = forward(tokens, plan, plan["positions"], None)
            best = binding.token_logprobs(logits, top=1)["top_id"][:, 0]
            out_tokens = [[int(best[cu[b + 1] - 1])] for b in range(B)]
            advance = new
            continue
        parent = sum([_tree.random_parents(rng, n) for n in ns], [])
        tokens = [int(x) for x in rng.integers(0, V, T)]
        for b in range(B):
            tokens[cu[b]] = out_tokens[b][-1]             # the root is the last emitted token
        tokens = i32(tokens)
        tree = binding.tree_plan(i32(parent + [0, 0]), plan["cu_new"], plan["kv_len"], words=1, status=plan["status"])
        logits = forward(tokens, plan, tree["positions"], tree["mask"])
        best = binding.token_logprobs(logits, tokens, top=1, status=None)["top_id"][:, 0].contiguous()
        # half of the drafts are made to be right, so that paths get long: the child's token is what was chosen
        for b in range(B):
            for i in range(1, ns[b]):
                if rng.random() < 0.5:
                    tokens[cu[b] + i] = best[cu[b] + parent[cu[b] + i]]
        logits = forward(tokens, plan, tree["positions"], tree["mask"])
        best = binding.token_logprobs(logits, top=1)["top_id"][:, 0].contiguous()
        keep = binding.tree_keep(i32(parent + [0, 0]), tokens, best, plan["cu_new"], plan["kv_len"], st["table"], st["kc"], st["vc"], max_out=8, status=plan["status"])
        advance = keep["n_out"]
        assert plan["status"].tolist() == [0] * B
        # ---- the host's view of the same round
        path = keep["path"].tolist()
        for b in range(B):
            way = path[b][:int(keep["n_out"][b])]
            assert way[0] == 0 and len(way) >= 1
            kept = [int(tokens[cu[b] + i]) for i in way]
            out_tokens[b] = keep["out_tokens"][b][:len(way)].tolist()
            assert kept[1:] == out_tokens[b][:-1]         # what the model chose behind a row is the next row's token
            hist[b] += kept
            # the kept tokens in a cache of their own, turned by their places in the sequence
            x = emb[i32(hist[b]).long()].view(-1, Hq + 2 * Hkv, D)
            n = len(hist[b])
            m = -(-n // page)
            kc1, vc1 = (torch.zeros(m, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
            q1 = binding.rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], i32(list(range(n))), freq, kc1, vc1, torch.arange(n, device="cuda"), q_weight=weights[0],
                                       k_weight=weights[1], eps=1e-6)
            pages = st["table"][b, :m].long()
            for cache, one in ((st["kc"], kc1), (st["vc"], vc1)):
                for layer in range(layers):
                    assert torch.equal(cache[layer, pages].flatten(0, 1)[:n], one.flatten(0, 1)[:n]), (step, b)
            # and its attention as a chain: the path's last row within both calls' bounds of the exact values
            ref = _paged.attention_reference(q1[-1:], kc1, vc1, torch.arange(m, dtype=torch.int32)[None], [0, 1], [n], 1 / 8)
            got, _ = binding.chunk_attention(q1[-1:].contiguous(), kc1, vc1, torch.arange(m, dtype=torch.int32, device="cuda")[None], i32([0, 1]), i32([n]))
            assert (np.abs(got.double().cpu().numpy() - ref[0]) <= ref[2]).all()
    assert sum(len(h) for h in hist) > 3 + 17 + 30 + 1 + 9 + 5 * B      # more was kept than the five roots of every request


def test_a_captured_round_over_trees_is_replayed(binding):
    """tree plan, rotation, attention, log probabilities and keep captured into one graph; replays equal eager calls on a copy."""
    B, n, Hq, Hkv, D, page, V = 4, 11, 8, 2, 128, 16, 5001
    rng = np.random.default_rng(5)
    g = torch.Generator().manual_seed(6)
    past = [30, 0, 77, 16]
    kv = [p + n for p in past]
    T = B * n
    W = 8
    table = torch.randperm(B * W, generator=g).to(torch.int32).view(B, W).cuda()
    slots = torch.tensor([int(table[b, p // page]) * page + p % page for b in range(B) for p in range(past[b], kv[b])], device="cuda")
    caches = [torch.randn(1, B * W, page, Hkv, D, generator=g).to(BF16).cuda() for _ in range(2)]
    copies = [c.clone() for c in caches]
    cu_t, kv_t = i32([n * b for b in range(B + 1)]), i32(kv)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(BF16).cuda()
    head = (torch.randn(Hq * D, V, generator=g) / 8).to(BF16).cuda()
    parent, tokens = i32([0] * T), i32([0] * T)
    freq = torch.rand(D // 2, generator=g).cuda()

    def round_(kc, vc):
        plan = binding.tree_plan(parent, cu_t, kv_t, words=1)
        q = binding.rotate_append(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], plan["positions"], freq, kc[0], vc[0], slots, eps=1e-6)
        o, l = binding.tree_attention(q, kc[0], vc[0], table, cu_t, kv_t, plan["mask"])
        lp = binding.token_logprobs(o.reshape(T, -1) @ head, tokens, top=3)
        keep = binding.tree_keep(parent, tokens, lp["top_id"][:, 0].contiguous(), cu_t, kv_t, table, kc, vc, max_out=5)
        return dict(lp, out=o, lse_attention=l, **keep)
    round_(*copies)
    for c, d in zip(caches, copies):
        d.copy_(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = round_(*caches)
    for step in range(10):
        qkv.copy_(torch.randn(T, Hq + 2 * Hkv, D, generator=g))
        parent.copy_(i32(sum([_tree.random_parents(rng, n) for _ in range(B)], [])))
        tokens.copy_(torch.randint(0, V, (T,), generator=g, dtype=torch.int32))
        graph.replay()
        want = round_(*copies)
        for k in want:
            assert torch.equal(got[k], want[k]), (step, k)
        assert all(torch.equal(a, b) for a, b in zip(caches, copies))


def test_calls_of_several_host_threads(binding):
    """Threads with a stream each, the operators at once: every result is what a call alone gives."""
    import threading
    lens = [(20, 900), (9, 40)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 40)
    q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
    mask = torch.tensor(_masks(np.random.default_rng(1), lens, "tree", 1)[0], device="cuda")
    x = torch.randn(7, 30000, generator=g).cuda()
    parent = i32(sum([_tree.random_parents(np.random.default_rng(2), n) for n, _ in lens], []))
    pos, freq, slot = i32(list(range(T))), torch.rand(64, generator=g).cuda(), torch.arange(T, device="cuda")
    jobs = [lambda s: binding.tree_attention(q, kc, vc, table, i32(cu), i32(kv), mask, stream=s), lambda s: tuple(binding.token_logprobs(x, top=9, stream=s).values()),
            lambda s: tuple(binding.tree_plan(parent, i32(cu), i32(kv), words=1, stream=s).values()),
            lambda s: (binding.rotate_append(q, q[:, :2], q[:, 2:4], pos, freq, torch.zeros_like(kc), torch.zeros_like(vc), slot, eps=1e-5, stream=s),),
            lambda s: tuple(binding.tree_keep(parent, parent, parent, i32(cu), i32(kv), max_out=4, stream=s).values())]
    want = [job(torch.cuda.current_stream()) for job in jobs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = jobs[i](s)
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
