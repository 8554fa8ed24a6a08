"""The paged cache's operators on the GPU against plain references (tests/_paged.py)."""
import math

import numpy as np
import pytest
import torch

from _paged import BAD_LEN, BAD_PAGE, BAD_POOL, NO_PAGES, NO_ROOM, attention_reference, build_cache, plan_reference

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


# ---- plan -----------------------------------------------------------------------------------------------------------
def _run_plan(binding, seq, adv, new, held, table, ring, ring_pos, page, max_tokens, in_place=False):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    t, r = torch.tensor(table, device="cuda"), torch.tensor(ring, device="cuda")
    s, h, rp = i32(seq), i32(held), torch.tensor(ring_pos, dtype=torch.int64, device="cuda")
    out = None
    if in_place:
        B = len(seq)
        out = {"seq_len": s, "pages_held": h, "ring_pos": rp, "cu_new": i32([7] * (B + 1)), "kv_len": i32([7] * B),
               "slot_map": torch.full((max_tokens,), 7, dtype=torch.int64, device="cuda"), "positions": i32([7] * max_tokens), "token_req": i32([7] * max_tokens),
               "status": i32([7] * B)}
    got = binding.cache_plan(s, i32(new), h, t, r, rp, page_size=page, max_tokens=max_tokens, advance=None if adv is None else i32(adv), out=out)
    return dict(got, block_table=t, free_ring=r)


def _check_plan(got, ref):
    for k, v in ref.items():
        assert np.array_equal(got[k].cpu().numpy(), np.asarray(v)), k


def _random_state(rng, B, page, W, spare, max_new=9):
    """Lengths, a table whose pages are all different, a ring with the rest at a random place."""
    seq = [int(rng.integers(0, W * page // 2)) for _ in range(B)]
    held = [min(W, -(-s // page) + int(rng.integers(0, 3))) for s in seq]
    P = sum(held) + spare
    perm = rng.permutation(P).astype(np.int32)
    table = np.full((B, W), -5, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    ring = np.full(P, -9, np.int32)
    head = int(rng.integers(0, 10 ** 12))
    for i in range(P - at):
        ring[(head + i) % P] = perm[at + i]
    adv = [int(rng.integers(-min(3, s), 5)) for s in seq]
    new = [int(rng.integers(-1, max_new)) for _ in range(B)]
    return seq, adv, new, held, table, ring, [head, head + P - at], P


@pytest.mark.parametrize("B,page,W,spare", [(1, 1, 40, 30), (1, 16, 8, 5), (3, 7, 9, 4), (33, 16, 20, 200), (257, 64, 6, 100), (1025, 8, 12, 4000), (8192, 16, 5, 20000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_matches_reference(binding, B, page, W, spare, in_place):
    rng = np.random.default_rng(B * 31 + page)
    seq, adv, new, held, table, ring, pos, P = _random_state(rng, B, page, W, spare)
    cap = sum(max(n, 0) for n in new) + 3
    ref = plan_reference(seq, adv, new, held, table, ring, pos, page, cap, P)
    _check_plan(_run_plan(binding, seq, adv, new, held, table, ring, pos, page, cap, in_place), ref)


@pytest.mark.parametrize("B,page,W,max_new", [(1, 24, 300, 6000), (5, 16, 400, 3000), (24, 64, 80, 2500), (200, 7, 60, 130), (513, 32, 12, 70), (2000, 16, 9, 40)])
def test_plan_of_long_chunks(binding, B, page, W, max_new):
    """Prompts among the chunks: slot maps of thousands of rows, over one and several CTAs and pages of any size."""
    rng = np.random.default_rng(B + page)
    seq, adv, new, held, table, ring, pos, P = _random_state(rng, B, page, W, B * (max_new // page + 2), max_new)
    for cap in (sum(max(n, 0) for n in new) + 700, sum(max(n, 0) for n in new) // 2):
        ref = plan_reference(seq, adv, new, held, table, ring, pos, page, cap, P)
        _check_plan(_run_plan(binding, seq, adv, new, held, table, ring, pos, page, cap), ref)


def test_plan_refusals_are_per_request(binding):
    """Too many tokens, too few pages, lengths that make no sense: each refused request says so, the others go on."""
    rng = np.random.default_rng(5)
    B, page, W = 40, 4, 16
    seq, adv, new, held, table, ring, pos, P = _random_state(rng, B, page, W, 6)
    new[3], new[5], held[7], held[8], adv[9], new[10] = -2, 10 ** 6, -1, W + 1, -10 ** 6, 2 ** 31 - 1
    seq[11] = 2 ** 31 - 1
    seen = set()
    hungry = [n + 30 if 0 < n < 100 else n for n in new]          # more pages than the pool has
    for asked in (new, hungry):
        for cap in (0, 1, 20, 60, 300, 2000):
            ref = plan_reference(seq, adv, asked, held, table, ring, pos, page, cap, P)
            _check_plan(_run_plan(binding, seq, adv, asked, held, table, ring, pos, page, cap), ref)
            for s in ref["status"]:
                seen |= {bit for bit in (BAD_LEN, NO_ROOM, NO_PAGES) if s & bit}
    assert seen == {BAD_LEN, NO_ROOM, NO_PAGES}


@pytest.mark.parametrize("pos", [[5, 4], [0, 10 ** 6], [-3, 2]])
def test_plan_bad_pool(binding, pos):
    rng = np.random.default_rng(6)
    seq, adv, new, held, table, ring, _, P = _random_state(rng, 9, 4, 16, 20)
    ref = plan_reference(seq, adv, new, held, table, ring, pos, 4, 50, P)
    got = _run_plan(binding, seq, adv, new, held, table, ring, pos, 4, 50)
    _check_plan(got, ref)
    assert all(s & BAD_POOL for s in got["status"].tolist())


def test_plan_bad_page_ids(binding):
    """Ids outside the pool, in the ring or in the table, give slot -1 and BAD_PAGE and are never followed."""
    rng = np.random.default_rng(8)
    seq, adv, new, held, table, ring, pos, P = _random_state(rng, 12, 4, 16, 60)
    new = [max(n, 1) for n in new]
    ring[pos[0] % P] = P
    ring[(pos[0] + 2) % P] = -1
    for b in range(6):
        p = seq[b] + adv[b]
        table[b, min(p // 4, 15)] = 2 ** 31 - 1
    ref = plan_reference(seq, adv, new, held, table, ring, pos, 4, 200, P)
    got = _run_plan(binding, seq, adv, new, held, table, ring, pos, 4, 200)
    _check_plan(got, ref)
    assert any(s & BAD_PAGE for s in ref["status"])


def test_plan_of_no_request(binding):
    got = _run_plan(binding, [], None, [], [], np.zeros((0, 3), np.int32), np.arange(4, dtype=np.int32), [1, 5], 4, 6)
    assert got["cu_new"].tolist() == [0] and got["slot_map"].tolist() == [-1] * 6 and got["ring_pos"].tolist() == [1, 5]


def test_plan_without_advance_and_strided_table(binding):
    rng = np.random.default_rng(9)
    seq, adv, new, held, table, ring, pos, P = _random_state(rng, 21, 16, 10, 40)
    ref = plan_reference(seq, [0] * 21, new, held, table, ring, pos, 16, 250, P)
    wide = torch.full((21, 17), -3, dtype=torch.int32, device="cuda")
    wide[:, :10] = torch.tensor(table, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    r = torch.tensor(ring, device="cuda")
    got = binding.cache_plan(i32(seq), i32(new), i32(held), wide[:, :10], r, torch.tensor(pos, device="cuda"), page_size=16, max_tokens=250)
    _check_plan(dict(got, block_table=wide[:, :10], free_ring=r), ref)
    assert (wide[:, 10:] == -3).all()


def test_plan_moves_every_page_of_the_largest_pool(binding):
    """A pool of 2^31 - 1 pages, all of them taken in one call and given back in the next: the counters of pages pass 2^31."""
    P, B, W = 2 ** 31 - 1, 8192, 2 ** 18
    ring = torch.arange(P, dtype=torch.int32, device="cuda")
    table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    i32 = lambda v: torch.full((B,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    seq = i32(W)
    seq[-1] = W - 1
    head = 12345
    got = binding.cache_plan(seq, i32(0), i32(0), table, ring, torch.tensor([head, head + P], device="cuda"), page_size=1, max_tokens=4096)
    assert (got["status"] == 0).all() and got["ring_pos"].tolist() == [head + P, head + P] and torch.equal(got["pages_held"], seq)
    flat, step = table.view(-1), 1 << 28
    for at in range(0, P, step):
        n = min(step, P - at)
        assert torch.equal(flat[at:at + n].long(), (torch.arange(at, at + n, device="cuda") + head) % P)
    assert int(flat[P]) == -1
    ring.fill_(-1)
    got = binding.cache_plan(got["seq_len"], i32(-1), got["pages_held"], table, ring, got["ring_pos"], page_size=1, max_tokens=4096)
    assert (got["status"] == 0).all() and got["ring_pos"].tolist() == [head + P, head + 2 * P] and (got["pages_held"] == 0).all()
    for at in range(0, P, step):       # in request order behind the ring's end, which has come round to place `head`
        n = min(step, P - at)
        assert torch.equal(ring[at:at + n].long(), torch.arange(at, at + n, device="cuda"))


def test_plans_of_several_host_threads(binding):
    """Plans of thousands of requests, of different sizes, called from several threads at once: none is refused, and each
    gives what it gives alone."""
    import ctypes as C
    import threading
    lib, jobs = binding.load_library(), []
    for B in (8192, 2100, 5000):
        rng = np.random.default_rng(B)
        seq, adv, new, held, table, ring, pos, P = _random_state(rng, B, 16, 5, 20000)
        cap = sum(max(n, 0) for n in new) + 3
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        t, r = torch.tensor(table, device="cuda"), torch.tensor(ring, device="cuda")
        args = [i32(seq), i32(new), i32(held), t, r, torch.tensor(pos, device="cuda"), i32(adv)]
        # (seq_len and the rest go to other arrays, so a call can be made again; what it moves then is not looked at)
        got = binding.cache_plan(*args[:6], page_size=16, max_tokens=cap, advance=args[6])
        _check_plan(dict(got, block_table=t, free_ring=r), plan_reference(seq, adv, new, held, table, ring, pos, 16, cap, P))
        d = binding.CachePlanDesc(B, 16, P, 5, cap, 5, *(x.data_ptr() for x in (args[0], args[6], args[1], args[2], args[5], t, r)),
                                  *(got[k].data_ptr() for k in ("seq_len", "pages_held", "ring_pos", "cu_new", "kv_len", "slot_map", "positions", "token_req", "status")))
        jobs.append((d, torch.cuda.Stream(), args, got))
    torch.cuda.synchronize()
    codes = [set() for _ in jobs]

    def work(i):
        d, stream, _, _ = jobs[i]
        for _ in range(3000):
            codes[i].add(lib.specsteer_cache_plan(C.byref(d), stream.cuda_stream))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert codes == [{binding.OK}] * len(jobs)


# ---- append ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,Hkv,D,page,dtype,layout", [
    (1, 1, 8, 1, BF16, "nhd"), (5, 8, 128, 16, BF16, "nhd"), (77, 2, 64, 32, F16, "hnd"), (33, 3, 80, 7, BF16, "hnd"), (40, 2, 33, 16, F16, "nhd"),
    (19, 4, 128, 64, torch.float32, "nhd"), (19, 1, 30, 5, torch.float32, "hnd"), (700, 8, 128, 16, BF16, "joined")])
def test_append_matches_indexing(binding, T, Hkv, D, page, dtype, layout):
    g = torch.Generator().manual_seed(T)
    P = -(-T // page) + 3
    mk = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    kc, vc = mk(P, page, Hkv, D).cuda(), mk(P, page, Hkv, D).cuda()
    if layout == "hnd":
        kc, vc = (c.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for c in (kc, vc))
    elif layout == "joined":
        pool = torch.stack((kc, vc), 1).contiguous()
        kc, vc = pool[:, 0], pool[:, 1]
    qkv = mk(T, 3, Hkv, D).cuda()
    k, v = qkv[:, 1], qkv[:, 2]                     # views into a fused projection's output
    slot = torch.randperm(P * page, generator=g)[:T].to(torch.int64)
    slot[::5] = -1
    if T > 3:
        slot[3] = P * page                          # just behind the cache
        slot[1] = 2 ** 40
    slot = slot.cuda()
    want_k, want_v = kc.clone(), vc.clone()
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < P * page:
            want_k[s // page, s % page], want_v[s // page, s % page] = k[t], v[t]
    binding.cache_append(k, v, kc, vc, slot)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_append_of_nothing(binding):
    kc, vc = torch.zeros(2, 4, 1, 8, device="cuda", dtype=BF16), torch.zeros(2, 4, 1, 8, device="cuda", dtype=BF16)
    e = torch.empty(0, 1, 8, device="cuda", dtype=BF16)
    binding.cache_append(e, e, kc, vc, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert (kc == 0).all()


# ---- attention ------------------------------------------------------------------------------------------------------
def _attend(binding, lens, Hq, Hkv, D, page, dtype, window=0, layout="nhd", seed=0, scale=None, generic=False, q_factor=1.0, extra_rows=3):
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", seed, layout, width_extra=seed % 3)
    q = (torch.randn(T + extra_rows, Hq, D, generator=g) * q_factor).to(dtype).cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full((T + extra_rows, Hq), 7.0, device="cuda")
    status = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got, got_lse = binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), scale=scale, window=window, out=out, lse=lse, status=status, generic=generic)
    assert got is out and got_lse is lse
    torch.cuda.synchronize()
    ref = attention_reference(q, kc, vc, table, cu, kv, 1.0 / math.sqrt(D) if scale is None else scale, window)
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
    # lens [(new, keys in all)], Hq, Hkv, D, page, dtype, window, layout
    ("one_token_one_key", [(1, 1)], 1, 1, 64, 16, BF16, 0, "nhd"),
    ("one_token", [(1, 1), (1, 129), (1, 2), (1, 500)], 8, 2, 128, 16, BF16, 0, "nhd"),
    ("chunk_of_five", [(5, 5), (5, 133), (5, 128), (5, 1027)], 16, 8, 128, 16, BF16, 0, "nhd"),
    ("idle_requests", [(0, 50), (3, 70), (0, 0), (6, 6), (0, 9)], 8, 1, 64, 32, F16, 0, "hnd"),
    ("rows_before_the_cache", [(9, 4), (3, 0), (5, 2)], 4, 2, 128, 16, BF16, 0, "nhd"),
    ("page_of_8", [(4, 77), (2, 260)], 4, 2, 64, 8, BF16, 0, "nhd"),
    ("page_of_128", [(7, 300), (7, 128), (1, 129)], 16, 2, 128, 128, F16, 0, "hnd"),
    ("page_of_256", [(5, 700), (2, 256)], 8, 2, 64, 256, BF16, 0, "nhd"),
    ("page_of_1", [(3, 40)], 2, 1, 64, 1, BF16, 0, "nhd"),
    ("page_of_24", [(5, 100), (1, 24)], 6, 2, 128, 24, BF16, 0, "nhd"),
    ("width_80", [(5, 200), (40, 200)], 6, 2, 80, 16, BF16, 0, "joined"),
    ("width_96", [(5, 200), (130, 150)], 4, 4, 96, 64, F16, 0, "nhd"),
    ("width_33", [(4, 60)], 4, 2, 33, 16, BF16, 0, "nhd"),
    ("width_8", [(4, 60), (1, 300), (200, 200)], 4, 2, 8, 16, F16, 0, "nhd"),
    ("width_40", [(5, 200), (130, 150)], 4, 2, 40, 64, BF16, 0, "hnd"),
    ("page_of_192", [(5, 700), (130, 385), (2, 192)], 8, 2, 128, 192, BF16, 0, "nhd"),
    ("group_of_128", [(3, 200)], 128, 1, 64, 16, BF16, 0, "nhd"),
    ("group_of_136", [(2, 70)], 136, 1, 64, 16, BF16, 0, "nhd"),
    ("window_past_all", [(5, 300), (1, 1)], 4, 2, 64, 16, BF16, 2 ** 31 - 1, "nhd"),
    ("width_256", [(3, 90), (20, 50)], 4, 2, 256, 16, BF16, 0, "nhd"),
    ("groups_of_5", [(5, 200), (60, 333)], 10, 2, 128, 16, BF16, 0, "nhd"),
    ("groups_of_7", [(9, 150), (50, 150)], 14, 2, 64, 16, BF16, 0, "hnd"),
    ("group_of_16", [(9, 400), (70, 400)], 16, 1, 128, 32, BF16, 0, "nhd"),
    ("group_of_40", [(2, 300)], 40, 1, 64, 16, BF16, 0, "nhd"),
    ("prompt", [(300, 300)], 4, 2, 128, 16, BF16, 0, "nhd"),
    ("prompt_chunks", [(129, 500), (257, 257), (1, 700), (256, 384)], 2, 1, 128, 64, BF16, 0, "nhd"),
    ("prompt_no_groups", [(513, 520)], 2, 2, 64, 32, F16, 0, "nhd"),
    ("window_1", [(5, 200), (1, 1), (40, 100)], 4, 2, 64, 16, BF16, 1, "nhd"),
    ("window_in_tile", [(5, 300), (200, 450)], 4, 2, 128, 16, BF16, 37, "nhd"),
    ("window_over_tiles", [(5, 900), (150, 700), (3, 100)], 8, 2, 128, 64, BF16, 300, "hnd"),
    ("many_requests", [(1 + i % 7, 1 + (i * 37) % 300 + i % 7) for i in range(90)], 4, 2, 64, 16, BF16, 0, "nhd"),
    ("long_context", [(5, 9001)], 4, 1, 128, 64, BF16, 0, "nhd"),
]


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("case", SHAPES, ids=[c[0] for c in SHAPES])
def test_attention_matches_reference(binding, case, generic):
    name, lens, Hq, Hkv, D, page, dtype, window, layout = case
    out, lse, status, ref = _attend(binding, lens, Hq, Hkv, D, page, dtype, window, layout, seed=len(name), generic=generic)
    _compare(out, lse, ref)
    assert (status == 0).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("factor,scale", [(12.0, None), (1.0, 0.0), (1.0, 3.0)])
def test_attention_sharp_and_flat_scores(binding, factor, scale, generic):
    """Scores of some tens (one key takes all the weight, the running maximum moves a lot) and a scale of zero."""
    out, lse, _, ref = _attend(binding, [(5, 700), (140, 300)], 4, 2, 128, 16, BF16, seed=4, scale=scale, q_factor=factor, generic=generic)
    _compare(out, lse, ref)


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_keys_a_row_does_not_see_do_not_reach_it(binding, generic):
    """NaN and infinities in keys and values of later positions: earlier rows are what they are without them; rows that
    see a NaN are NaN where it belongs."""
    for lens, window in (([(6, 200), (130, 260)], 0), ([(6, 200), (130, 260)], 50)):
        kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 3)
        q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        spots = {0: (197, float("nan"), float("inf")), 1: (200, float("inf"), float("nan"))}
        for b, (j, kx, vx) in spots.items():
            page = int(table[b, j // 16])
            kc[page, j % 16, 1, 5] = kx
            vc[page, j % 16, 0, 77] = vx
        out, lse = binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), window=window, generic=generic)
        o = out.float().cpu()
        ref = attention_reference(q, kc, vc, table, cu, kv, 1 / math.sqrt(128), window)
        for b, (n, total) in enumerate(lens):
            j = spots[b][0]
            for i in range(n):
                p = total - n + i
                sees = j <= p and (not window or j > p - window)
                row = o[cu[b] + i]
                clean = row.clone()
                if sees:
                    assert not torch.isfinite(row[:4, 77]).any()          # kv head 0: the spoilt value, its column alone
                    clean[:4, 77] = 0
                    if math.isnan(spots[b][1]):
                        assert not torch.isfinite(row[4:]).any()          # kv head 1: the spoilt key
                    clean[4:] = 0                                         # (an infinite score may also be -inf: weight 0)
                assert torch.isfinite(clean).all(), (b, i, sees)
                if not sees:
                    err = np.abs(row.double().numpy() - ref[0][cu[b] + i])
                    assert (err <= ref[2][cu[b] + i]).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_bad_lengths_and_pages(binding, generic):
    lens = [(5, 100), (4, 90), (6, 300), (3, 60)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 64, BF16, "cuda", 11)
    q = torch.randn(T, 4, 64, generator=g).to(BF16).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table[2, 1], table[2, 7] = kc.shape[0], -1
    table[2, 18] = 2 ** 31 - 1
    for kv_bad, cu_bad in ((kv[:1] + [-1] + kv[2:], cu), (kv[:1] + [table.shape[1] * 16 + 1] + kv[2:], cu), (kv[:1] + [2 ** 31 - 1] + kv[2:], cu)):
        out, lse = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda")
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        binding.chunk_attention(q, kc, vc, table, i32(cu_bad), i32(kv_bad), out=out, lse=lse, status=status, generic=generic)
        assert status.tolist() == [0, BAD_LEN, BAD_PAGE, 0]
        ref = attention_reference(q, kc, vc, table, cu_bad, kv_bad, 1 / 8)
        _compare(out, lse, ref)
    # offsets that go down, or past the rows of q
    for cu_bad, want in (([0, 5, 3, 15, T], [0, BAD_LEN, BAD_PAGE, 0]), ([0, 5, 9, 15, T + 1], [0, 0, BAD_PAGE, BAD_LEN]), ([-1, 5, 9, 15, T], [BAD_LEN, 0, BAD_PAGE, 0])):
        out, lse = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda")
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        binding.chunk_attention(q, kc, vc, table, i32(cu_bad), i32(kv), out=out, lse=lse, status=status, generic=generic)
        assert status.tolist() == want


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("cu_bad", [[0, 5, 9, 15, 19], [-1, 5, 9, 15, 18], [5, 9, 2, 2, 5], [0, 5, 5, 2 ** 31 - 1, 18], [3, 3, -2 ** 31, 15, 18]])
def test_attention_offsets_that_make_no_sense(binding, cu_bad, generic):
    """Requests with offsets past the rows, before them or going down write nothing, and the others are what they are alone.
    (No row belongs to two of the accepted requests.)"""
    lens = [(5, 100), (4, 90), (6, 300), (3, 60)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 64, BF16, "cuda", 15)
    assert T == 18
    q = torch.randn(T, 4, 64, generator=g).to(BF16).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse, status = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda"), i32([0] * 4)
    binding.chunk_attention(q, kc, vc, table, i32(cu_bad), i32(kv), out=out, lse=lse, status=status, generic=generic)
    bad = [a < 0 or b < a or b > T for a, b in zip(cu_bad, cu_bad[1:])]
    assert any(bad) and not all(bad)
    assert status.tolist() == [BAD_LEN * x for x in bad]
    _compare(out, lse, attention_reference(q, kc, vc, table, cu_bad, kv, 1 / 8))


def test_attention_strided_q_and_out(binding):
    """q inside a fused projection's output, out a slice of a wider buffer, a stride that is no multiple of 16 bytes."""
    lens = [(5, 100), (130, 200)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 12)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    fused = torch.randn(T, 12 * 128, generator=g).to(BF16).cuda()
    for q in (fused[:, :1024].view(T, 8, 128), torch.randn(T, 8, 131, generator=g).to(BF16).cuda()[..., 1:129]):
        buf = torch.full((T, 8, 200), 7.0, dtype=BF16, device="cuda")
        out, lse = binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), out=buf[..., 3:131])
        ref = attention_reference(q, kc, vc, table, cu, kv, 1 / math.sqrt(128))
        _compare(out, lse, ref)
        assert (buf[..., :3] == 7).all() and (buf[..., 131:] == 7).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("above", [100.0, 140.0, 200.0, 300.0])
def test_attention_one_key_far_above_those_before_it(binding, above, generic):
    """A key anywhere in a block of keys whose score is a hundred or more above every score so far takes all the weight."""
    kc, vc, table, cu, kv, T, g = build_cache([(1, 900)] * 64 + [(3, 640)] * 2, 16, 1, 64, BF16, "cuda", 21)
    kc[torch.isfinite(kc)] = 0
    for b in range(66):
        j = 576 + b % 64
        kc[int(table[b, j // 16]), j % 16, 0, 0] = above
    q = torch.zeros(T, 2, 64, dtype=BF16, device="cuda")
    q[..., 0] = 1
    out, lse = torch.full_like(q, 7.0), torch.full((T, 2), 7.0, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), scale=1.0, out=out, lse=lse, generic=generic)
    _compare(out, lse, attention_reference(q, kc, vc, table, cu, kv, 1.0))


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("dtype,size,scale", [(F16, 40.0, 1.0), (F16, 4000.0, 0.088), (F16, 8000.0, 1.0), (F16, 60000.0, 1.0), (F16, 60000.0, 1e9), (BF16, 1e5, 1.0), (BF16, 3e6, 0.125),
                                              (BF16, 1e12, 1.0), (BF16, 1e19, 0.01), (BF16, 1e19, 30.0), (BF16, 1.0, 1e38), (BF16, 1e-3, 1e38)])
def test_attention_very_large_scores(binding, dtype, size, scale, generic):
    """Scores of up to 1e38 and scales of up to 1e38: the largest key takes all the weight, keys of the same score share it.

    Only one column of q and k is not zero, so that every score is one product of two numbers of 11 bits, exact in float32.
    The keys below the largest are 0.1 size or more below it, so their scores are 0.05 size^2 scale (80 or more) below, their
    weights less than 2^-115 of its, and the result is the mean of the values of the two largest, whose weights are alike.
    What is left is the rounding of the result (u of it), of the weights to the inputs' type for the product with v (u of the
    mean of |v|: the weight is 2^x with an x that carries half a step of the scaled maximum, so it need not be a power of
    two), and 2^-20 for the division and the joining of parts."""
    lens = [(1, 900), (5, 700), (1, 1), (150, 400), (3, 9001), (1, 130)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 64, dtype, "cpu", 70)
    used = torch.isfinite(kc)
    kc[used] = 0
    for b, (n, total) in enumerate(lens):
        x = size * (2 * torch.rand(total, 2, generator=g) - 1) * 0.8
        top = torch.randint(0, max(1, total - n), (2,), generator=g)
        x[top] = size * (0.9 + 0.1 * torch.rand(1, 2, generator=g))              # both of the largest alike, seen by every row
        for j in range(total):
            kc[int(table[b, j // 16]), j % 16, :, 0] = x[j].to(dtype)
    q = torch.zeros(T, 8, 64, dtype=dtype)
    q[..., 0] = (size * (0.5 + 0.5 * torch.rand(T, 8, generator=g))).to(dtype)
    q, kc, vc, table = (t.cuda() for t in (q, kc, vc, table))
    out, lse = torch.full_like(q, 7.0), torch.full((T, 8), 7.0, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), scale=scale, out=out, lse=lse, generic=generic)
    want, want_lse, _, _, written = attention_reference(q, kc, vc, table, cu, kv, float(np.float32(scale)))
    assert written.all() and np.isfinite(want).all()
    u = torch.finfo(dtype).eps / 2
    tol = np.abs(want) * u + np.abs(vc[torch.isfinite(vc)].double().cpu().numpy()).max() * (u * (1 + u) + 2.0 ** -20) + (2.0 ** -25 if dtype == F16 else 0.0)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    with np.errstate(over="ignore", invalid="ignore"):
        want_lse = want_lse.astype(np.float32).astype(np.float64)                # (beyond float32: infinite)
        got = lse.double().cpu().numpy()
        assert ((got == want_lse) | (np.abs(got - want_lse) <= 8 * 2.0 ** -24 * np.abs(want_lse))).all()


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_many_small_weights_of_float16(binding, generic):
    """In every 128 keys one that takes nearly all the weight, with value 0, and 127 of 2^-25.2 of its weight, which are all
    that the result consists of.

    With the weights held 2^8 up, a weight below float16's normal range is off by 2^-25 against a largest one of 2^8, so
    the reference's term for it shrinks by 2^8."""
    n = 1280
    kc, vc, table, cu, kv, T, g = build_cache([(1, n)], 64, 1, 64, F16, "cuda", 22)
    used = torch.isfinite(kc)
    kc[used], vc[used] = 0, 100.0
    for j in range(0, n, 128):
        page = int(table[0, j // 64])
        kc[page, 0, 0, 0] = 17.5
        vc[page, 0] = 0
    q = torch.zeros(T, 1, 64, dtype=F16, device="cuda")
    q[..., 0] = 1
    out, lse = torch.full_like(q, 7.0), torch.full((T, 1), 7.0, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), scale=1.0, out=out, lse=lse, generic=generic)
    want, want_lse, tol, tol_lse, written = attention_reference(q, kc, vc, table, cu, kv, 1.0)
    tol = tol - n * 2.0 ** -25 * 100.0 * (1 - 2.0 ** -8)
    assert want.min() > 2e-4 and tol.max() < 2e-5
    _compare(out, lse, (want, want_lse, tol, tol_lse, written))


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_tiny_scale(binding, generic):
    """Huge queries and keys with a scale that brings their products back to ordinary scores, and one that makes them nothing."""
    kc, vc, table, cu, kv, T, g = build_cache([(5, 300), (1, 200)], 16, 2, 64, BF16, "cuda", 23)
    kc *= 3e17
    q = (torch.randn(T, 4, 64, generator=g) * 3e17).to(BF16).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for scale in (1e-35, 0.0):
        out, lse = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda")
        binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), scale=scale, out=out, lse=lse, generic=generic)
        _compare(out, lse, attention_reference(q, kc, vc, table, cu, kv, float(np.float32(scale))))


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
@pytest.mark.parametrize("page", [8, 16, 64, 128])
def test_attention_pages_behind_the_window_may_be_gone(binding, page, generic):
    """With a window, pages that no row sees any more can have been given back: their entries are not looked at."""
    lens, window = [(5, 700), (1, 90), (150, 600), (3, 333)], 70
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, 2, 64, BF16, "cuda", 60)
    for b, (n, total) in enumerate(lens):
        table[b, :max(0, total - n + 1 - window) // page] = -1
    assert (table[0] == -1).any() and (table[2] == -1).any()
    q = torch.randn(T, 8, 64, generator=g).to(BF16).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse, status = torch.full_like(q, 7.0), torch.full((T, 8), 7.0, device="cuda"), i32([0] * 4)
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), window=window, out=out, lse=lse, status=status, generic=generic)
    _compare(out, lse, attention_reference(q, kc, vc, table, cu, kv, 1 / 8, window))
    assert status.tolist() == [0] * 4


# With the blocks of 64 keys that 148 CTAs load on average: a CTA that has as many or more stops before them.
STOP_SHAPES = [
    ("one_tile_parts", [(5, 60001), (0, 9), (3, 700)], 8, 1, 128, 64, BF16, (0, 2, 4)),                     # 938 / 148 = 6.3
    ("two_tiles", [(2500, 2500), (700, 3900), (1, 5)], 8, 2, 128, 16, BF16, (0, 2, 5, 12)),                 # 64 tokens a unit: 2870 / 148 = 19
    ("single_tokens", [(1, 1 + 97 * i) for i in range(60)], 8, 4, 64, 32, F16, (0, 2, 5, 12)),              # 10700 / 148 = 72
    ("windows_of_whole_units", [(300, 2000)] * 3 + [(5, 900)] * 40, 16, 4, 64, 8, F16, (0, 2, 4)),          # 1040 / 148 = 7.0
]


@pytest.mark.parametrize("case", STOP_SHAPES, ids=[c[0] for c in STOP_SHAPES])
def test_attention_waits_that_run_out_are_reported(binding, case):
    """CTAs that stop loading keys after some blocks: the waits for the next ones run out (after a second), the kernel ends by
    itself and says TIMEOUT on request 0, and the call after it is what it was before.  Rows of no request, and those of refused
    requests, are left as they are."""
    name, lens, Hq, Hkv, D, page, dtype, stops = case
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", 80)
    q = torch.randn(T + 3, Hq, D, generator=g).to(dtype).cuda()
    kv[2] = -1
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    args = (q, kc, vc, table, i32(cu), i32(kv))
    mine = torch.ones(T + 3, dtype=torch.bool, device="cuda")
    mine[T:] = False
    mine[cu[2]:cu[3]] = False

    def call(**k):
        out, lse, status = torch.full_like(q, 7.0), torch.full((T + 3, Hq), 7.0, device="cuda"), i32([0] * len(lens))
        binding.chunk_attention(*args, out=out, lse=lse, status=status, window=300 if name.startswith("window") else 0, **k)
        torch.cuda.synchronize()
        assert (out[~mine] == 7).all() and (lse[~mine] == 7).all()
        assert int(status[2]) == BAD_LEN and int(status.sum()) - int(status[0]) == BAD_LEN
        return out, lse, int(status[0])
    want, want_lse, status = call()
    assert status == 0
    for blocks in stops:
        out, lse, status = call(stop_after=blocks)
        assert status == binding.REQ_TIMEOUT
        out, lse, status = call()
        assert status == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
    out, lse, status = call(stop_after=65534)             # more than any CTA has
    assert status == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("case", STOP_SHAPES, ids=[c[0] for c in STOP_SHAPES])
def test_attention_that_gave_up_leaves_nan(binding, case):
    """A caller who passes no status sees a wait that ran out too: every row of the accepted requests is NaN, no other row is."""
    name, lens, Hq, Hkv, D, page, dtype, stops = case
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", 81)
    q = torch.randn(T + 3, Hq, D, generator=g).to(dtype).cuda()
    kv[2] = -1
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    mine = torch.ones(T + 3, dtype=torch.bool, device="cuda")
    mine[T:] = False
    mine[cu[2]:cu[3]] = False
    wide = torch.full((T + 3, Hq, D + 16), 7.0, dtype=dtype, device="cuda")
    out, lse = wide[..., 8:8 + D], torch.full((T + 3, Hq), 7.0, device="cuda")
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), out=out, lse=lse, stop_after=stops[-1])
    assert out[mine].isnan().all() and lse[mine].isnan().all()
    assert (out[~mine] == 7).all() and (lse[~mine] == 7).all() and (wide[..., :8] == 7).all() and (wide[..., 8 + D:] == 7).all()


@pytest.mark.parametrize("seed", range(32))
def test_attention_random_shapes(binding, seed):
    """Shapes, lengths, windows, layouts and bad pages drawn at random over what the tensor-core kernel takes."""
    rng = np.random.default_rng(1000 + seed)
    pick = lambda *v: v[int(rng.integers(len(v)))]  # noqa: E731
    Hkv, G, D, page = pick(1, 2, 3), pick(1, 2, 3, 4, 5, 8, 12, 16), 8 * int(rng.integers(1, 17)), pick(8, 16, 32, 64, 128, 192)
    dtype, window, layout = pick(BF16, F16), pick(0, 0, int(rng.integers(1, 300))), pick("nhd", "hnd", "joined")
    lens = []
    for _ in range(int(rng.integers(1, 7))):
        n = pick(0, 1, int(rng.integers(1, 10)), int(rng.integers(1, 90)), int(rng.integers(1, 400 // G + 2)))
        lens.append((n, max(0, n + pick(-2, 0, int(rng.integers(0, 130)), int(rng.integers(0, 700))))))
    kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", seed, layout, width_extra=seed % 2)
    want = []
    for b, (n, total) in enumerate(lens):
        first = max(0, total - n + 1 - window) if window else 0
        used = list(range(first // page, -(-total // page))) if n and total > 0 else []
        if used and rng.random() < 0.3:
            table[b, used[int(rng.integers(len(used)))]] = pick(-1, kc.shape[0], 2 ** 31 - 1, -2 ** 31)
            want.append(BAD_PAGE)
        else:
            want.append(0)
    q = torch.randn(T + 2, Hkv * G, D, generator=g).to(dtype).cuda()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse, status = torch.full_like(q, 7.0), torch.full((T + 2, Hkv * G), 7.0, device="cuda"), i32([0] * len(lens))
    binding.chunk_attention(q, kc, vc, table, i32(cu), i32(kv), window=window, out=out, lse=lse, status=status)
    with np.errstate(invalid="ignore"):
        _compare(out, lse, attention_reference(q, kc, vc, table, cu, kv, 1 / math.sqrt(D), window))
    assert status.tolist() == want


def test_attention_same_bits_again_and_beside_other_work(binding):
    lens = [(5, 2000), (5, 70), (1, 900), (300, 700)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 13)
    q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
    cu_t, kv_t = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cu, kv))
    first, lse = binding.chunk_attention(q, kc, vc, table, cu_t, kv_t)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s in streams:
            got.append(binding.chunk_attention(q, kc, vc, table, cu_t, kv_t, stream=s))
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, first) and torch.equal(l, lse)


def test_attention_refuses_small_workspace_and_bad_arguments(binding):
    lens = [(5, 100)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 14)
    q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
    cu_t, kv_t = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cu, kv))
    with pytest.raises(ValueError):
        binding.chunk_attention(q.half(), kc, vc, table, cu_t, kv_t)
    with pytest.raises(ValueError):
        binding.chunk_attention(q, kc, vc, table, cu_t, kv_t[:0])
    with pytest.raises(ValueError):
        binding.chunk_attention(q, kc, vc, table.long(), cu_t, kv_t)
    for bad in (dict(scale=-1.0), dict(scale=float("inf")), dict(window=-1)):
        with pytest.raises(binding.SpecSteerError) as e:
            binding.chunk_attention(q, kc, vc, table, cu_t, kv_t, **bad)
        assert e.value.code == binding.ERR_INVALID_ARG
    with pytest.raises(binding.SpecSteerError) as e:
        binding.chunk_attention(q[:, :7], kc, vc, table, cu_t, kv_t)          # 7 heads over 2
    assert e.value.code == binding.ERR_INVALID_ARG


def test_attention_workspaces_that_do_not_serve(binding):
    lens = [(5, 100)]
    kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", 14)
    q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
    cu_t, kv_t = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cu, kv))
    want, want_lse = binding.chunk_attention(q, kc, vc, table, cu_t, kv_t)
    room = torch.empty(200 << 20, dtype=torch.uint8, device="cuda")
    got, lse = binding.chunk_attention(q, kc, vc, table, cu_t, kv_t, workspace=room[64:])
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    for bad in (room[:1 << 20], room[8:], room[:0]):
        with pytest.raises(binding.SpecSteerError) as e:
            binding.chunk_attention(q, kc, vc, table, cu_t, kv_t, workspace=bad)
        assert e.value.code == binding.ERR_WORKSPACE
    binding.chunk_attention(q, kc, vc, table, cu_t, kv_t, workspace=room[:0], generic=True)     # needs none


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_cache_beyond_32_bit_offsets(binding, generic):
    """Pools of more than 2^31 elements, of which only the last pages are used."""
    P, page, Hkv, D, n, kv = 140_000, 16, 8, 128, 6, 150
    kc, vc = (torch.empty(P, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
    assert kc.numel() > 2 ** 31
    g = torch.Generator().manual_seed(31)
    pages = [P - 1 - 3 * i for i in range(-(-kv // page))]
    table = torch.tensor([pages], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(kv, Hkv, D, generator=g).to(BF16) for _ in range(2))
    slots = torch.tensor([pages[i // page] * page + i % page for i in range(kv)], device="cuda")
    binding.cache_append(k.cuda(), v.cuda(), kc, vc, slots)
    assert torch.equal(kc[pages[0], :, 3].cpu(), k[:page, 3]) and torch.equal(vc[pages[-1], 0].cpu(), v[(len(pages) - 1) * page])
    vc[pages[-1], (kv - 1) % page, 2, 9] = float("inf")          # seen by the last row alone
    v[kv - 1, 2, 9] = 0
    q = torch.randn(n, 16, D, generator=g).to(BF16).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse = binding.chunk_attention(q, kc, vc, table, i32([0, n]), i32([kv]), generic=generic)
    assert torch.isposinf(out[n - 1, 4:6, 9]).all() and torch.isposinf(out).sum() == 2
    out[n - 1, 4:6, 9] = 0
    ref = list(attention_reference(q, k[None], v[None], torch.zeros(1, 1, dtype=torch.int32), [0, n], [kv], 1 / math.sqrt(D)))
    ref[0][n - 1, 4:6, 9] = 0
    _compare(out, lse, ref)


@pytest.mark.parametrize("generic", [False, True], ids=["", "generic"])
def test_attention_thousands_of_requests(binding, generic):
    """More requests than a block has threads several times over, many of them idle."""
    lens = [((0, 1, 0, 3, 1)[i % 5], (i * 7) % 45 + 3) for i in range(5001)]
    out, lse, status, ref = _attend(binding, lens, 2, 1, 64, 16, BF16, seed=32, generic=generic)
    _compare(out, lse, ref)
    assert (status == 0).all()


def test_calls_of_several_host_threads(binding):
    """Threads with a stream each, different shapes at once: every result is what a call alone gives."""
    import threading
    cases = []
    for i, (lens, Hq, Hkv, D, page, dtype) in enumerate([([(5, 900), (5, 30)], 8, 2, 128, 16, BF16), ([(1, 700)] * 9, 4, 4, 64, 32, F16), ([(200, 300)], 4, 1, 96, 64, BF16), ([(3, 90)], 2, 1, 200, 16, BF16)]):
        kc, vc, table, cu, kv, T, g = build_cache(lens, page, Hkv, D, dtype, "cuda", 40 + i)
        q = torch.randn(T, Hq, D, generator=g).to(dtype).cuda()
        args = (q, kc, vc, table) + tuple(torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cu, kv))
        cases.append((args, binding.chunk_attention(*args)))
    torch.cuda.synchronize()
    wrong = []

    def work(args, want):
        s = torch.cuda.Stream()
        for _ in range(30):
            out, lse = binding.chunk_attention(*args, stream=s)
            s.synchronize()
            if not (torch.equal(out, want[0]) and torch.equal(lse, want[1])):
                wrong.append(args[0].shape)
    threads = [threading.Thread(target=work, args=c) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_two_captured_calls_replayed_at_once(binding):
    """Two graphs of the attention, each with a workspace of its own, replayed on two streams at the same time."""
    graphs = []
    for seed, lens in ((50, [(5, 3000), (5, 40)]), (51, [(150, 900)])):
        kc, vc, table, cu, kv, T, g = build_cache(lens, 16, 2, 128, BF16, "cuda", seed)
        q = torch.randn(T, 8, 128, generator=g).to(BF16).cuda()
        args = (q, kc, vc, table) + tuple(torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cu, kv))
        want = binding.chunk_attention(*args)
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            got = binding.chunk_attention(*args)
        graphs.append((graph, stream, args, want, got))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream, *_ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, _, want, got in graphs:
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# ---- a run of them together -------------------------------------------------------------------------------------------
def _loop_state(B, page, W, P, seed):
    g = torch.Generator().manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"seq_len": i32([0] * B), "held": i32([0] * B), "table": torch.full((B, W), -1, dtype=torch.int32, device="cuda"),
            "ring": torch.randperm(P, generator=g).to(torch.int32).cuda(), "pos": torch.tensor([0, P], device="cuda")}


def test_rounds_with_a_cache_on_the_device(binding):
    """Prompt, then rounds: plan -> append -> attention -> verify -> plan with the round's n_out, nothing read back in
    between.  Every chunk's attention equals attention over the tokens kept so far, held in plain lists on the host."""
    from paper_2603_16219_b200 import synth
    B, K, Hq, Hkv, D, page, W, P = 6, 3, 8, 2, 64, 16, 12, 60
    st = _loop_state(B, page, W, P, 1)
    g = torch.Generator().manual_seed(2)
    kc = torch.full((P, page, Hkv, D), float("nan"), dtype=BF16, device="cuda")
    vc = kc.clone()
    spec = synth.RoundSpec("loop", B, K, 4001, "f32", ragged=True, temp_choices=(0.7, 1.0))
    ctx = binding.Context(B, K, 4001)
    prompts = [1, 17, 64, 5, 33, 90]
    hist = [[] for _ in range(B)]                       # per request the (k, v) of every token kept
    advance, new = None, torch.tensor(prompts, dtype=torch.int32, device="cuda")
    for step in range(5):
        cap = sum(prompts) if step == 0 else B * (K + 1)
        plan = binding.cache_plan(st["seq_len"], new, st["held"], st["table"], st["ring"], st["pos"], page_size=page, max_tokens=cap, advance=advance)
        st.update(seq_len=plan["seq_len"], held=plan["pages_held"], pos=plan["ring_pos"])
        q, k, v = (torch.randn(cap, h, D, generator=g).to(BF16).cuda() for h in (Hq, Hkv, Hkv))
        binding.cache_append(k, v, kc, vc, plan["slot_map"])
        out, lse = binding.chunk_attention(q, kc, vc, st["table"], plan["cu_new"], plan["kv_len"], status=plan["status"])
        inputs = synth.make_round(spec, device="cuda", seed=step)
        outs = binding.verify_recover_round(ctx, inputs, flags=binding.FLAG_BONUS)
        # ---- host's view of the same step
        cu, kv = plan["cu_new"].tolist(), plan["kv_len"].tolist()
        assert plan["status"].tolist() == [0] * B
        for b in range(B):
            hist[b] += [(k[i].cpu(), v[i].cpu()) for i in range(cu[b], cu[b + 1])]
            assert len(hist[b]) == kv[b]
            n = cu[b + 1] - cu[b]
            flat_k, flat_v = (torch.stack([t[x] for t in hist[b]])[None] for x in (0, 1))       # one page that holds it all
            ref = attention_reference(q[cu[b]:cu[b + 1]], flat_k, flat_v, torch.zeros(1, 1, dtype=torch.int32), [0, n], [kv[b]], 1 / 8)
            _compare(out[cu[b]:cu[b + 1]], lse[cu[b]:cu[b + 1]], ref)
            keep = n if step == 0 else int(outs["n_out"][b])
            del hist[b][kv[b] - n + min(keep, n):]
        pages = [st["table"][b, :int(st["held"][b])].tolist() for b in range(B)]
        flat = sum(pages, []) + [int(st["ring"][i % P]) for i in range(int(st["pos"][0]), int(st["pos"][1]))]
        assert sorted(flat) == list(range(P))            # every page is in one table or in the ring
        if step == 0:
            advance = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        else:
            advance = torch.minimum(outs["n_out"], inputs["draft_len"] + 1)
        new = synth.make_round(spec, device="cuda", seed=step + 1)["draft_len"] + 1
    ctx.close()


def test_a_captured_round_is_replayed(binding):
    """plan, append and attention captured into a graph, in place; replays equal eager calls on a copy of the state."""
    B, n, Hq, Hkv, D, page, W, P = 5, 4, 8, 2, 128, 16, 40, 90
    st = _loop_state(B, page, W, P, 3)
    g = torch.Generator().manual_seed(4)
    T = B * n
    kc, vc = (torch.randn(P, page, Hkv, D, generator=g).to(BF16).cuda() for _ in range(2))
    q, k, v = (torch.randn(T, h, D, generator=g).to(BF16).cuda() for h in (Hq, Hkv, Hkv))
    new = torch.full((B,), n, dtype=torch.int32, device="cuda")
    adv = torch.tensor([4, 1, 3, 2, 4], dtype=torch.int32, device="cuda")
    copies = [t.clone() for t in (st["seq_len"], st["held"], st["table"], st["ring"], st["pos"], kc, vc)]

    def buffers(seq, held, pos):
        e = lambda m, dt=torch.int32: torch.empty(m, dtype=dt, device="cuda")  # noqa: E731
        return {"seq_len": seq, "pages_held": held, "ring_pos": pos, "cu_new": e(B + 1), "kv_len": e(B), "slot_map": e(T, torch.int64), "positions": e(T),
                "token_req": e(T), "status": e(B)}

    def round_(seq, held, table, ring, pos, kc, vc, out, o, l):
        plan = binding.cache_plan(seq, new, held, table, ring, pos, page_size=page, max_tokens=T, advance=adv, out=out)
        binding.cache_append(k, v, kc, vc, plan["slot_map"])
        binding.chunk_attention(q, kc, vc, table, plan["cu_new"], plan["kv_len"], out=o, lse=l, status=plan["status"])

    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    l1, l2 = (torch.empty(T, Hq, device="cuda") for _ in range(2))
    warm = [t.clone() for t in copies]
    round_(*warm[:5], *warm[5:], buffers(warm[0], warm[1], warm[4]), o1, l1)
    out1 = buffers(st["seq_len"], st["held"], st["pos"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_(st["seq_len"], st["held"], st["table"], st["ring"], st["pos"], kc, vc, out1, o1, l1)
    out2 = buffers(copies[0], copies[1], copies[4])
    for step in range(40):
        q.copy_(torch.randn(T, Hq, D, generator=g))
        graph.replay()
        round_(*copies[:5], *copies[5:], out2, o2, l2)
        assert torch.equal(o1, o2) and torch.equal(l1, l2) and torch.equal(st["table"], copies[2]) and torch.equal(kc, copies[5])
        for name in out1:
            assert torch.equal(out1[name], out2[name]), name
    assert out1["seq_len"].tolist() == [40 * a for a in adv.tolist()]
