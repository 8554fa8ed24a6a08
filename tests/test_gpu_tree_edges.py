"""A round over trees of drafts on the GPU: arguments at the ends of what the operators accept, and the attention inside a run of rounds."""
import ctypes as C

import numpy as np
import pytest
import torch

import _paged
import _tree

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- rotate ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("D,rot,dtype", [(64, 64, BF16), (128, 64, F32), (24, 8, F16), (33, 32, BF16), (40, 6, F32)])
def test_rotate_weights_belong_to_the_norm(binding, D, rot, dtype, neighbours):
    """A descriptor without a norm (eps < 0) whose weights are given all the same: no norm, and so no weights, whichever kernel takes it."""
    T, Hq, Hkv, page = 9, 4, 2, 16
    g = torch.Generator().manual_seed(D)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
    pos, freq, slot = torch.arange(T, dtype=torch.int32), torch.rand(rot // 2, generator=g), torch.arange(T)
    weight = torch.full((D,), 3.0).cuda()
    kc, vc = (torch.zeros(1, page, Hkv, D, dtype=dtype, device="cuda") for _ in range(2))
    out = torch.empty(T, Hq, D, dtype=dtype, device="cuda")
    tok, row, es = qkv.stride(0), page * Hkv * D, qkv.element_size()
    pos_d, freq_d, slot_d = pos.cuda(), freq.cuda(), slot.cuda()
    d = binding.RotateAppendDesc(T, Hq, Hkv, D, rot, 1, int(neighbours), page, 1, binding._CACHE_DTYPES[dtype], binding.F32, -1.0, 1.0, tok, D, tok, D, tok, D, Hq * D, D, row, Hkv * D, D,
                                 row, Hkv * D, D, qkv.data_ptr(), qkv.data_ptr() + Hq * D * es, qkv.data_ptr() + (Hq + Hkv) * D * es, out.data_ptr(), weight.data_ptr(),
                                 weight.data_ptr(), pos_d.data_ptr(), freq_d.data_ptr(), None, slot_d.data_ptr(), kc.data_ptr(), vc.data_ptr())
    assert binding.load_library().specsteer_rotate_append(d, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == binding.OK
    for got, x in ((out, qkv[:, :Hq]), (kc[0, :T], qkv[:, Hq:Hq + Hkv])):
        want, tol = _tree.rotate_reference(x, None, None, [pos.tolist()], freq, None, neighbours, 1.0)
        assert ((got.double().cpu() - want).abs() <= tol).all()


# ---- log probabilities ----------------------------------------------------------------------------------------------
def _check_logprobs(binding, x, temperature, top):
    """The definition in 64 bits, rounded to float32 (log probabilities beyond its range are -inf).  The bounds are those of
    _tree.logprobs_reference; that of a log probability counts log sum exp(l - max l) from the largest one, which is its negative,
    because the largest l may be too large for float64 to hold the two's sum."""
    R, V = x.shape
    tokens = torch.arange(0, V, max(1, V // 50), dtype=torch.int32).repeat(R, 1)
    status = i32([0] * R)
    got = binding.token_logprobs(x.cuda(), tokens.cuda(), temperature=temperature.cuda(), top=top, status=status)
    assert (status == 0).all()
    logp, lse, entropy, tol_lse, tol_h, _ = _tree.logprobs_reference(x, temperature)
    e = 2.0 ** -24
    log_s = -logp.max(1).values
    p = logp.exp()
    mean = torch.where(p > 0, p * (-log_s[:, None] - logp), torch.zeros_like(p)).sum(1)
    tol_p = 256 * e + 2.0 ** -22 + 5 * e * mean + 2.0 ** -22 + 6 * e * log_s
    assert ((got["lse"].double().cpu() - lse).abs() <= tol_lse).all()
    assert ((got["entropy"].double().cpu() - entropy).abs() <= tol_h).all()
    ids = _tree.top_reference(x, top)
    assert torch.equal(got["top_id"].long().cpu(), ids)
    for name, lp in (("logprob", logp.gather(1, tokens.long())), ("top_logprob", logp.gather(1, ids))):
        a, gone = got[name].double().cpu(), torch.isneginf(lp.float())
        assert torch.equal(torch.isneginf(a), gone), name
        assert ((a - lp).abs() <= tol_p[:, None] + 6 * e * lp.abs())[~gone].all(), name


SIZES = [(6, 700), (6, 40003), (760, 5003), (900, 700)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,V", SIZES)
def test_logprobs_of_tiny_temperatures(binding, R, V, dtype):
    """Temperatures down to the least float32, over logits of their size (a largest logit of 0 among them), with rows that begin with
    huge negative ones: lse is finite, and so is everything else."""
    temp = torch.tensor([2.0 ** -149, 1e-43, 1e-39, 4.2e-39, 2.0 ** -126, 3e-38]).repeat(R // 6 + 1)[:R]
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(R, V, generator=g).double() * 5 * temp.double()[:, None]).to(dtype)
    x[::2] = -x[::2].abs()
    x[::2, V // 3::7] = 0
    x[2::3, :V // 2] = -1e35 if dtype != F16 else -60000.0
    x[::5, ::9] = torch.finfo(dtype).min
    x[::7, 1::9] = -INF
    _check_logprobs(binding, x, temp, 20)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,V", SIZES)
def test_logprobs_of_logits_a_range_apart(binding, R, V, dtype):
    """Logits from the type's lowest value to its largest, whose differences pass float32's range, under temperatures from 1 to the largest."""
    temp = torch.tensor([3.4e38, 1e37, 2e38, 5.0, 1.0, 1e30]).repeat(R // 6 + 1)[:R]
    g = torch.Generator().manual_seed(V)
    x = ((torch.rand(R, V, generator=g) * 2 - 1) * torch.finfo(dtype).max).to(dtype)
    x[:, ::11], x[:, 5::13] = torch.finfo(dtype).min, torch.finfo(dtype).max / 2
    x[::2, V - 1] = torch.finfo(dtype).max
    x[2::3, :V // 2] = torch.finfo(dtype).min
    x[::7, 1::9] = -INF
    _check_logprobs(binding, x, temp, 20)


# ---- a run of rounds ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("sampled", [False, True], ids=["likeliest", "sampled"])
@pytest.mark.parametrize("window", [0, 11])
def test_attention_inside_rounds(binding, window, sampled):
    """Rounds over trees, whose path rows are compared layer by layer with chains of the same tokens: queries, keys and values bit by bit, the
    attention's output with the definition over the chain.  Tokens are chosen as the likeliest ones, or sampled and steered by a
    round without drafts (K = 0) over the rows."""
    B, Hq, Hkv, D, page, W, P, layers, V = 4, 8, 2, 64, 16, 14, 50, 2, 97
    g, rng = torch.Generator().manual_seed(5), np.random.default_rng(6)
    ring, ring_pos = torch.randperm(P, generator=g).to(torch.int32).cuda(), torch.tensor([0, P], device="cuda")
    seq_len, held, table = i32([0] * B), i32([0] * B), torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    kc, vc = (torch.full((layers, P, page, Hkv, D), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
    emb = torch.randn(layers, V, (Hq + 2 * Hkv) * D, generator=g).to(BF16).cuda()   # a token's projections in every layer
    head = (torch.randn(Hq * D, V, generator=g) / 2).to(BF16).cuda()
    other = torch.randn(2, V, generator=g).cuda()                                   # stands for the specialist's logits
    freq = (1e4 ** (-torch.arange(D // 2) / (D // 2))).cuda()
    norm = dict(q_weight=torch.rand(D, generator=g).cuda() + 0.5, k_weight=torch.rand(D, generator=g).cuda() + 0.5, eps=1e-6)
    ctx = binding.Context(B * 20 + 2, 0, V) if sampled else None

    def split(x):
        x = x.view(-1, Hq + 2 * Hkv, D)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    def forward(tokens, plan, positions, mask):
        qs, outs = [], []
        for layer in range(layers):
            q = binding.rotate_append(*split(emb[layer][tokens.long()]), positions, freq, kc[layer], vc[layer], plan["slot_map"], **norm)
            args = (q, kc[layer], vc[layer], table, plan["cu_new"], plan["kv_len"])
            if mask is None:
                o, _ = binding.chunk_attention(*args, window=window, status=plan["status"])
            else:
                o, _ = binding.tree_attention(*args, mask, positions=positions, window=window, status=plan["status"])
            qs.append(q)
            outs.append(o)
        return qs, outs, sum(o.reshape(len(o), -1).nan_to_num(0) for o in outs) @ head

    def choose(logits):
        if not sampled:
            return binding.token_logprobs(logits, top=1)["top_id"][:, 0].contiguous()
        T = len(logits)
        h = logits.float().view(T, 1, V)
        u = torch.rand(T, generator=g).cuda()
        none_f, ones = torch.empty(T, 0, device="cuda"), torch.ones(T, device="cuda")
        got = binding.verify_recover_round(ctx, dict(h_llm=h, h_slm_plus=other[0].expand(T, 1, V).contiguous(), h_slm_minus=other[1].expand(T, 1, V).contiguous(),
                                                     draft_tokens=torch.empty(T, 0, dtype=torch.int32, device="cuda"), draft_len=i32([0] * T), lam=ones, beta=ones * 0.5,
                                                     temperature=ones, u_accept=none_f, u_recover=u), flags=binding.FLAG_BONUS)
        # the sample is that of the steered law: the smallest token whose cumulated probability passes u, but for the roundings of a
        # cumulated probability: 97 additions to 2^-24 and weights to 2^-22 in all, less than 1e-5
        p = torch.softmax(h[:, 0].double() + 0.5 * (other[0].double() - other[1].double()), 1).cumsum(1)
        tok = got["rec_token"].long()
        upper = p.gather(1, tok[:, None])[:, 0]
        lower = torch.where(tok > 0, p.gather(1, (tok - 1).clamp(min=0)[:, None])[:, 0], 0.0)
        assert (upper > u.double() - 1e-5).all() and (lower < u.double() + 1e-5).all() and (got["n_out"] == 1).all()
        return got["rec_token"]

    hist = [[int(x) for x in rng.integers(0, V, n)] for n in (3, 17, 30, 1)]
    last, advance, longer = None, None, 0
    for step in range(4):
        ns = [len(h) for h in hist] if step == 0 else [1 + int(rng.integers(0, 20)) for _ in range(B)]
        T = sum(ns) + 2
        plan = binding.cache_plan(seq_len, i32(ns), held, table, ring, ring_pos, page_size=page, max_tokens=T, advance=advance)
        seq_len, held, ring_pos = plan["seq_len"], plan["pages_held"], plan["ring_pos"]
        cu = plan["cu_new"].tolist()
        if step == 0:
            _, _, logits = forward(i32(sum(hist, []) + [0, 0]), plan, plan["positions"], None)
            best = choose(logits)
            last, advance = [int(best[cu[b + 1] - 1]) for b in range(B)], i32(ns)
            continue
        parent = i32(sum([_tree.random_parents(rng, n) for n in ns], []) + [0, 0])
        tokens = i32([int(x) for x in rng.integers(0, V, T)])
        for b in range(B):
            tokens[cu[b]] = last[b]
        tree = binding.tree_plan(parent, plan["cu_new"], plan["kv_len"], words=1, window=window, status=plan["status"])
        # drafts that are right for one choice of the rows above them: two thirds, so that paths get long
        state = g.get_state()
        best = choose(forward(tokens, plan, tree["positions"], tree["mask"])[2])
        for b in range(B):
            for i in range(1, ns[b]):
                if rng.random() < 0.67:
                    tokens[cu[b] + i] = best[cu[b] + int(parent[cu[b] + i])]
        g.set_state(state)                                # (the same uniforms again)
        qs, outs, logits = forward(tokens, plan, tree["positions"], tree["mask"])
        best = choose(logits)
        keep = binding.tree_keep(parent, tokens, best, plan["cu_new"], plan["kv_len"], table, kc, vc, max_out=8, status=plan["status"])
        advance = keep["n_out"]
        assert plan["status"].tolist() == [0] * B
        for b in range(B):
            way = keep["path"][b, :int(keep["n_out"][b])].tolist()
            rows = torch.tensor([cu[b] + i for i in way], device="cuda")
            emitted, past = keep["out_tokens"][b, :len(way)].tolist(), len(hist[b])
            assert way[0] == 0 and emitted == best[rows].tolist() and tokens[rows[1:]].tolist() == emitted[:-1]
            hist[b] += tokens[rows].tolist()
            last[b] = emitted[-1]
            longer += len(way) - 1
            n = len(hist[b])
            m = -(-n // page)
            pages, own = table[b, :m].long(), torch.arange(m, dtype=torch.int32)[None]
            for layer in range(layers):
                kc1, vc1 = (torch.zeros(m, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
                q1 = binding.rotate_append(*split(emb[layer][i32(hist[b]).long()]), i32(list(range(n))), freq, kc1, vc1, torch.arange(n, device="cuda"), **norm)
                assert torch.equal(qs[layer][rows], q1[past:])
                for cache, one in ((kc, kc1), (vc, vc1)):
                    assert torch.equal(cache[layer, pages].flatten(0, 1)[:n], one.flatten(0, 1)[:n])
                want = _paged.attention_reference(q1[past:], kc1, vc1, own, [0, n - past], [n], 1 / 8, window)
                err = np.abs(outs[layer][rows].double().cpu().numpy() - want[0])
                assert (err <= want[2]).all(), (step, b, layer, (err / want[2]).max())
    assert longer >= 5                                    # paths of more than the root, whose rows hang on drafted ones
