"""Descriptors and host-side refusals of the operators of a round over trees of drafts: nothing here needs a GPU."""
import ctypes as C
import os
import re
import struct

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 4096   # a pointer that is not NULL and 32-byte aligned; every call below is refused before anything is launched


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


DESCS = [("tree_plan", "TreePlanDesc"), ("rotate_append", "RotateAppendDesc"), ("tree_attention", "TreeAttentionDesc"), ("token_logprobs", "TokenLogprobsDesc"),
         ("tree_keep", "TreeKeepDesc")]


@pytest.mark.parametrize("name,mirror", DESCS)
def test_descriptor_layout_matches_header(binding, name, mirror):
    hdr = open(os.path.join(ROOT, "include", "specsteer.h")).read()
    end = hdr.index("} specsteer_%s_desc;" % name)
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.rindex("typedef struct {", 0, end) + len("typedef struct {"):end], flags=re.S)
    fields, types = [], []
    for decl in body.split(";"):
        decl = decl.strip()
        if not decl:
            continue
        kind = decl.split()[1 if decl.startswith("const") else 0]
        for part in decl.split(","):
            fields.append(re.findall(r"([A-Za-z_0-9]+)\s*$", part.strip())[0])
            types.append("P" if "*" in decl else {"int32_t": "i", "int64_t": "q", "float": "f", "specsteer_attention_desc": "a"}[kind])
    cls = getattr(binding, mirror)
    assert fields == [n for n, _ in cls._fields_]
    code = {C.c_int32: "i", C.c_int64: "q", C.c_float: "f", C.c_void_p: "P", binding.AttentionDesc: "a"}
    assert types == [code[t] for _, t in cls._fields_]
    assert struct.Struct("@" + binding._codes(cls)).size == C.sizeof(cls)      # what the calls pack


def _desc(cls, base, k):
    d = cls()
    for name, typ in cls._fields_:
        if typ is C.c_void_p:
            setattr(d, name, PTR)
    for name, v in {**base, **k}.items():
        setattr(d, name, v)
    return d


def _call(binding, name, mirror, base, k):
    return getattr(binding.load_library(), "specsteer_" + name)(_desc(getattr(binding, mirror), base, k), None)


PLAN = dict(B=2, T=9, mask_words=2, window=0, ld_mask=2)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(T=-1), dict(mask_words=0), dict(mask_words=33), dict(ld_mask=1), dict(window=-1), dict(parent=None), dict(cu_new=None),
                                 dict(kv_len=None), dict(mask=None), dict(B=2 ** 31 - 1)])
def test_plan_refuses(binding, bad):
    assert _call(binding, "tree_plan", "TreePlanDesc", PLAN, bad) == binding.ERR_INVALID_ARG
    assert binding.load_library().specsteer_tree_plan(None, None) == binding.ERR_INVALID_ARG
    assert _call(binding, "tree_plan", "TreePlanDesc", PLAN, dict(B=0, T=0, parent=None, mask=None, kv_len=None)) == binding.OK


ROT = dict(T=3, Hq=4, Hkv=2, D=64, rot=64, n_axes=1, neighbours=0, page_size=16, n_pages=8, dtype=1, weight_dtype=0, eps=-1.0, factor=1.0, q_tok=256, q_head=64, k_tok=128,
           k_head=64, v_tok=128, v_head=64, o_tok=256, o_head=64, kc_page=2048, kc_slot=128, kc_head=64, vc_page=2048, vc_slot=128, vc_head=64)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(Hq=-1), dict(Hkv=-1), dict(D=0), dict(rot=66), dict(rot=-2), dict(rot=3), dict(n_axes=0), dict(page_size=0), dict(n_pages=0),
                                 dict(dtype=3), dict(weight_dtype=-1), dict(eps=float("nan")), dict(factor=float("nan")), dict(q_tok=-1), dict(vc_head=-8), dict(o_tok=0),
                                 dict(o_head=0), dict(kc_page=0), dict(vc_slot=0), dict(kc_head=0), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slot_map=None),
                                 dict(k_cache=None), dict(positions=None), dict(inv_freq=None)])
def test_rotate_refuses(binding, bad):
    assert _call(binding, "rotate_append", "RotateAppendDesc", ROT, bad) == binding.ERR_INVALID_ARG
    assert binding.load_library().specsteer_rotate_append(None, None) == binding.ERR_INVALID_ARG


def test_rotate_limits(binding):
    assert _call(binding, "rotate_append", "RotateAppendDesc", ROT, dict(D=binding.ROTATE_MAX_D + 2)) == binding.ERR_UNSUPPORTED
    for nothing in (dict(T=0, q=None, k=None, positions=None), dict(Hq=0, Hkv=0, q=None, k=None, slot_map=None, k_cache=None)):
        assert _call(binding, "rotate_append", "RotateAppendDesc", ROT, nothing) == binding.OK


ATT = dict(B=2, T=4, Hq=4, Hkv=2, D=64, page_size=16, n_pages=8, table_width=4, dtype=1, window=0, scale=0.125, flags=0, ld_table=4, q_tok=256, q_head=64, o_tok=256, o_head=64,
           kc_page=2048, kc_slot=128, kc_head=64, vc_page=2048, vc_slot=128, vc_head=64, workspace_bytes=0)


def _tree(binding, a=None, **k):
    base = dict(a=_desc(binding.AttentionDesc, ATT, a or {}), mask_words=1, ld_mask=1)
    return _desc(binding.TreeAttentionDesc, base, k)


def test_attention_refuses(binding):
    fn = binding.load_library().specsteer_tree_attention
    assert fn(None, None) == binding.ERR_INVALID_ARG
    for bad in (dict(B=-1), dict(Hq=5), dict(D=0), dict(window=-1), dict(dtype=0), dict(q=None), dict(out=None), dict(o_tok=0), dict(scale=2.4e38), dict(flags=2)):
        assert fn(_tree(binding, a=bad), None) == binding.ERR_INVALID_ARG, bad
    for bad in (dict(mask_words=0), dict(ld_mask=0), dict(mask=None), dict(mask_words=2)):
        assert fn(_tree(binding, **bad), None) == binding.ERR_INVALID_ARG, bad
    assert fn(_tree(binding, a=dict(window=5), positions=None), None) == binding.ERR_INVALID_ARG
    assert fn(_tree(binding, a=dict(D=257)), None) == binding.ERR_UNSUPPORTED
    assert fn(_tree(binding, a=dict(workspace=None)), None) == binding.ERR_WORKSPACE
    assert fn(_tree(binding, a=dict(T=0), mask=None), None) == binding.OK


LOG = dict(R=3000, V=100, n_tokens=1, n_top=5, dtype=1, ld_row=100, ld_tok=1, workspace_bytes=1 << 30)


@pytest.mark.parametrize("bad", [dict(R=-1), dict(V=0), dict(n_tokens=-1), dict(n_top=-1), dict(n_top=33), dict(V=4, ld_row=4), dict(ld_row=99), dict(dtype=3), dict(ld_tok=0),
                                 dict(logits=None), dict(token=None), dict(logprob=None), dict(top_id=None), dict(top_logprob=None)])
def test_logprobs_refuses(binding, bad):
    lib = binding.load_library()
    assert _call(binding, "token_logprobs", "TokenLogprobsDesc", LOG, bad) == binding.ERR_INVALID_ARG
    assert lib.specsteer_token_logprobs(None, None) == binding.ERR_INVALID_ARG and lib.specsteer_token_logprobs_workspace(None) == 0


def test_logprobs_workspace(binding):
    lib = binding.load_library()
    need = lib.specsteer_token_logprobs_workspace(_desc(binding.TokenLogprobsDesc, LOG, {}))
    assert need > 0
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=PTR + 16)):
        assert _call(binding, "token_logprobs", "TokenLogprobsDesc", LOG, bad) == binding.ERR_WORKSPACE
    assert _call(binding, "token_logprobs", "TokenLogprobsDesc", LOG, dict(R=0, logits=None, workspace=None)) == binding.OK
    assert lib.specsteer_token_logprobs_workspace(_desc(binding.TokenLogprobsDesc, LOG, dict(R=0))) == 0


KEEP = dict(B=2, T=9, max_out=4, n_layers=3, Hkv=2, D=64, page_size=16, n_pages=8, table_width=4, dtype=1, ld_table=4, kc_layer=1 << 14, kc_page=2048, kc_slot=128, kc_head=64,
            vc_layer=1 << 14, vc_page=2048, vc_slot=128, vc_head=64)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(T=-1), dict(max_out=0), dict(n_layers=-1), dict(Hkv=0), dict(D=0), dict(page_size=0), dict(n_pages=0), dict(table_width=0),
                                 dict(ld_table=3), dict(dtype=3), dict(kc_layer=0), dict(kc_page=0), dict(vc_slot=0), dict(vc_head=0), dict(kc_slot=-1), dict(parent=None),
                                 dict(token=None), dict(choice=None), dict(cu_new=None), dict(kv_len=None), dict(block_table=None), dict(k_cache=None), dict(v_cache=None),
                                 dict(n_out=None), dict(Hkv=1 << 16, D=1 << 16)])
def test_keep_refuses(binding, bad):
    assert _call(binding, "tree_keep", "TreeKeepDesc", KEEP, bad) == binding.ERR_INVALID_ARG
    assert binding.load_library().specsteer_tree_keep(None, None) == binding.ERR_INVALID_ARG
    assert _call(binding, "tree_keep", "TreeKeepDesc", KEEP, dict(B=0, cu_new=None, n_out=None)) == binding.OK


def test_binding_checks_tensors(binding):
    import torch
    i32, bf = torch.int32, torch.bfloat16
    par, cu, kv = torch.zeros(9, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    mask, pos = torch.zeros(9, 2, dtype=i32), torch.zeros(9, dtype=i32)
    for call in (lambda: binding.tree_plan(par.long(), cu, kv, words=2), lambda: binding.tree_plan(par, cu[:2], kv, words=2), lambda: binding.tree_plan(par, cu, kv, words=0),
                 lambda: binding.tree_plan(par, cu, kv, words=1, out={"mask": mask, "positions": pos}), lambda: binding.tree_plan(par, cu, kv, words=2 ** 32 + 1),
                 lambda: binding.tree_plan(par, cu, kv, words=2, out={"mask": mask[:8], "positions": pos}), lambda: binding.tree_plan(par, cu, kv, words=2, window=2 ** 31)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):                      # no CPU fallback
        binding.tree_plan(par, cu, kv, words=2)
    table = torch.zeros(2, 4, dtype=i32)
    kc, q = torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(9, 4, 64, dtype=bf)
    for call in (lambda: binding.tree_attention(q, kc, kc, table, cu, kv, mask[:8]), lambda: binding.tree_attention(q, kc, kc, table, cu, kv, mask.long()),
                 lambda: binding.tree_attention(q, kc, kc, table, cu, kv, mask, window=5), lambda: binding.tree_attention(q, kc, kc, table, cu, kv, mask.t()[:1].t()[:, :0]),
                 lambda: binding.tree_attention(q, kc, kc, table, cu, kv, mask, positions=pos[:3], window=5), lambda: binding.tree_attention(q.half(), kc, kc, table, cu, kv, mask)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        binding.tree_attention(q, kc, kc, table, cu, kv, mask)
    k, slot, fr = torch.zeros(9, 2, 64, dtype=bf), torch.zeros(9, dtype=torch.int64), torch.zeros(32)
    w = torch.zeros(64)
    rot = binding.rotate_append
    for call in (lambda: rot(q, k, k, pos, fr, kc, kc, slot[:8]), lambda: rot(q, k[:8], k, pos, fr, kc, kc, slot), lambda: rot(q.half(), k, k, pos, fr, kc, kc, slot),
                 lambda: rot(q, k, k, pos[:8], fr, kc, kc, slot), lambda: rot(q, k, k, pos.long(), fr, kc, kc, slot), lambda: rot(q, k, k, pos, fr.double(), kc, kc, slot),
                 lambda: rot(q, k, k, pos, fr, kc, kc, slot, q_weight=w), lambda: rot(q, k, k, pos, fr, kc, kc, slot, eps=-1.0),
                 lambda: rot(q, k, k, pos, fr, kc, kc, slot, eps=1e-6, q_weight=w, k_weight=w.to(bf)), lambda: rot(q, k, k, pos, fr, kc, kc, slot, eps=1e-6, q_weight=w.double()),
                 lambda: rot(q, k, k, pos, fr, kc, kc, slot, axis_of=torch.zeros(31, dtype=i32)), lambda: rot(q[..., :32], k, k, pos, fr, kc, kc, slot),
                 lambda: rot(q, k, k, pos, fr, kc, kc, slot, eps=1e-6, q_weight=w[:32])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        rot(q, k, k, pos, fr, kc, kc, slot)
    lg, tok = torch.zeros(3, 50), torch.zeros(3, dtype=i32)
    lp = binding.token_logprobs
    for call in (lambda: lp(lg[0]), lambda: lp(lg.double()), lambda: lp(lg.t()), lambda: lp(lg, tok[:2]), lambda: lp(lg, tok.long()), lambda: lp(lg, tok[0]), lambda: lp(lg, tok.view(3, 1, 1)), lambda: lp(lg, top=33), lambda: lp(lg, top=-1),
                 lambda: lp(lg[:, :4], top=5), lambda: lp(lg, temperature=torch.zeros(2)), lambda: lp(lg, status=torch.zeros(3))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        lp(lg, tok, top=3)
    keep = binding.tree_keep
    for call in (lambda: keep(par, par[:8], par, cu, kv, max_out=3), lambda: keep(par, par, par, cu, kv, max_out=0), lambda: keep(par, par, par, cu, kv, table, kc, max_out=3),
                 lambda: keep(par, par, par, cu, kv, None, kc, kc, max_out=3), lambda: keep(par, par, par, cu, kv, table[:1], kc, kc, max_out=3),
                 lambda: keep(par, par, par, cu, kv, table, kc, kc.half(), max_out=3), lambda: keep(par, par, par, cu, kv, table, kc[0], kc[0], max_out=3),
                 lambda: keep(par, par, par, cu, kv, table, max_out=3), lambda: keep(par, par, par, cu, kv, max_out=2 ** 31)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        keep(par, par, par, cu, kv, table, kc, kc, max_out=3)


def test_binding_refuses_a_stream_of_another_device(binding):
    import types

    import torch
    i32, bf = torch.int32, torch.bfloat16
    par, cu, kv, pos = torch.zeros(9, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(9, dtype=i32)
    kc, q, k = torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(9, 4, 64, dtype=bf), torch.zeros(9, 2, 64, dtype=bf)
    other = types.SimpleNamespace(device_index=1)
    for call in (lambda: binding.tree_plan(par, cu, kv, words=2, stream=other), lambda: binding.tree_keep(par, par, par, cu, kv, max_out=2, stream=other),
                 lambda: binding.tree_attention(q, kc, kc, torch.zeros(2, 4, dtype=i32), cu, kv, torch.zeros(9, 1, dtype=i32), stream=other),
                 lambda: binding.rotate_append(q, k, k, pos, torch.zeros(32), kc, kc, torch.zeros(9, dtype=torch.int64), stream=other),
                 lambda: binding.token_logprobs(torch.zeros(3, 50), stream=other)):
        with pytest.raises(ValueError, match="stream"):
            call()


def test_the_reference_climbs_and_packs(binding):
    """The references that the GPU tests compare with, on a tree worked out by hand."""
    import numpy as np
    import torch

    import _tree
    #      0 -> 1, 2;  1 -> 3;  3 -> 4
    mask, pos, status = _tree.plan_reference([-1, 0, 0, 1, 3], [0, 5], [12], 6, 1)
    assert mask[:, 0].tolist() == [1, 3, 5, 11, 27, 0] and pos == [7, 8, 8, 9, 10, -1] and status == [0]
    assert _tree.plan_reference([-1, 0, 0, 1, 3], [0, 5], [12], 5, 1, window=2)[0][:, 0].tolist() == [1, 3, 5, 10, 24]
    seen = np.zeros((40, 40), bool)
    seen[3, 31] = seen[3, 32] = True
    assert _tree.pack_bits(seen, 2)[3].tolist() == [-2 ** 31, 1]
    got = _tree.keep_reference([-1, 0, 0, 1, 3], [5, 6, 7, 8, 9], [7, 8, 1, 9, 2], [0, 5], [12], 5, 4)
    assert got[:3] == ([2], [[0, 2, -1, -1]], [[7, 1, -1, -1]]) and got[4] == [0]
    logp, lse, h, *_ = _tree.logprobs_reference(torch.zeros(1, 8))
    assert abs(lse.item() - np.log(8)) < 1e-12 and abs(h.item() - np.log(8)) < 1e-12
