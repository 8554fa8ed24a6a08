"""Descriptors and host-side refusals of the paged cache's operators: nothing here needs a GPU."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


@pytest.mark.parametrize("name,mirror,size", [("cache_plan", "CachePlanDesc", 6 * 4 + 8 + 16 * 8), ("cache_append", "CacheAppendDesc", 6 * 4 + 15 * 8),
                                              ("attention", "AttentionDesc", 12 * 4 + 11 * 8 + 11 * 8)])
def test_descriptor_layout_matches_header(binding, name, mirror, size):
    hdr = open(os.path.join(ROOT, "include", "specsteer.h")).read()
    end = hdr.index("} specsteer_%s_desc;" % name)
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.rindex("typedef struct {", 0, end) + len("typedef struct {"):end], flags=re.S)
    fields = []
    for decl in body.split(";"):
        for part in decl.strip().split(","):
            if part.strip():
                fields.append(re.findall(r"([A-Za-z_0-9]+)\s*$", part.strip())[0])
    cls = getattr(binding, mirror)
    assert fields == [n for n, _ in cls._fields_]
    assert C.sizeof(cls) == size


PTR = 4096   # a pointer that is not NULL; every call below is refused before anything is launched


def _plan(binding, **k):
    d = binding.CachePlanDesc(B=2, page_size=16, n_pages=8, table_width=4, max_tokens=10, ld_table=4)
    for name, typ in d._fields_:
        if typ is C.c_void_p:
            setattr(d, name, PTR)
    for name, v in k.items():
        setattr(d, name, v)
    return d


def _append(binding, **k):
    d = binding.CacheAppendDesc(T=2, Hkv=2, D=64, page_size=16, n_pages=8, dtype=binding.BF16, k_tok=128, k_head=64, v_tok=128, v_head=64, kc_page=2048, kc_slot=128,
                                kc_head=64, vc_page=2048, vc_slot=128, vc_head=64, k=PTR, v=PTR, slot_map=PTR, k_cache=PTR, v_cache=PTR)
    for name, v in k.items():
        setattr(d, name, v)
    return d


def _attention(binding, **k):
    d = binding.AttentionDesc(B=2, T=4, Hq=4, Hkv=2, D=64, page_size=16, n_pages=8, table_width=4, dtype=binding.BF16, window=0, scale=0.125, ld_table=4,
                              q_tok=256, q_head=64, o_tok=256, o_head=64, kc_page=2048, kc_slot=128, kc_head=64, vc_page=2048, vc_slot=128, vc_head=64,
                              q=PTR, k_cache=PTR, v_cache=PTR, block_table=PTR, cu_new=PTR, kv_len=PTR, out=PTR)
    for name, v in k.items():
        setattr(d, name, v)
    return d


@pytest.mark.parametrize("bad", [dict(B=-1), dict(page_size=0), dict(n_pages=0), dict(table_width=0), dict(max_tokens=-1), dict(ld_table=3), dict(seq_len=None),
                                 dict(new_len=None), dict(pages_held=None), dict(ring_pos=None), dict(block_table=None), dict(free_ring=None), dict(seq_len_out=None),
                                 dict(pages_held_out=None), dict(ring_pos_out=None), dict(cu_new=None), dict(kv_len=None), dict(slot_map=None), dict(req_status=None)])
def test_plan_refuses(binding, bad):
    assert binding.load_library().specsteer_cache_plan(_plan(binding, **bad), None) == binding.ERR_INVALID_ARG


def test_plan_refuses_too_many_requests(binding):
    assert binding.load_library().specsteer_cache_plan(_plan(binding, B=binding.PLAN_MAX_B + 1), None) == binding.ERR_UNSUPPORTED
    assert binding.load_library().specsteer_cache_plan(None, None) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(T=-1), dict(Hkv=0), dict(D=0), dict(page_size=0), dict(n_pages=0), dict(dtype=3), dict(dtype=-1), dict(k=None), dict(v=None),
                                 dict(slot_map=None), dict(k_cache=None), dict(v_cache=None), dict(k_tok=-1), dict(vc_head=-8), dict(Hkv=1 << 16, D=1 << 16)])
def test_append_refuses(binding, bad):
    assert binding.load_library().specsteer_cache_append(_append(binding, **bad), None) == binding.ERR_INVALID_ARG
    assert binding.load_library().specsteer_cache_append(None, None) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(B=-1), dict(T=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=5), dict(D=0), dict(page_size=0), dict(n_pages=0), dict(table_width=0),
                                 dict(ld_table=3), dict(dtype=0), dict(dtype=7), dict(window=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(flags=2), dict(q_tok=-1), dict(o_head=-1), dict(kc_page=-1), dict(q=None), dict(k_cache=None), dict(v_cache=None),
                                 dict(block_table=None), dict(cu_new=None), dict(kv_len=None), dict(out=None)])
def test_attention_refuses(binding, bad):
    lib = binding.load_library()
    assert lib.specsteer_chunk_attention(_attention(binding, **bad), None) == binding.ERR_INVALID_ARG
    assert lib.specsteer_chunk_attention_workspace(_attention(binding, **bad)) == 0


def test_attention_refuses_wide_heads_and_takes_nothing(binding):
    lib = binding.load_library()
    assert lib.specsteer_chunk_attention(_attention(binding, D=binding.ATTENTION_MAX_D + 1), None) == binding.ERR_UNSUPPORTED
    assert lib.specsteer_chunk_attention(None, None) == binding.ERR_INVALID_ARG
    for d in (_attention(binding, T=0, q=None, out=None), _attention(binding, B=0, cu_new=None)):
        assert lib.specsteer_chunk_attention(d, None) == binding.OK
    assert lib.specsteer_cache_append(_append(binding, T=0, k=None), None) == binding.OK


def test_attention_refuses_a_scale_that_does_not_fit_powers_of_two(binding):
    """The kernels weigh with powers of two: scale * log2(e) has to be a float32 too (scale up to 2.35e38)."""
    lib = binding.load_library()
    assert lib.specsteer_chunk_attention(_attention(binding, scale=2.4e38), None) == binding.ERR_INVALID_ARG
    assert lib.specsteer_chunk_attention(_attention(binding, scale=2.3e38, T=0, q=None, out=None), None) == binding.OK


def test_binding_checks_tensors(binding):
    import torch
    i32 = torch.int32
    seq, ring, pos = torch.zeros(2, dtype=i32), torch.zeros(8, dtype=i32), torch.zeros(2, dtype=torch.int64)
    table = torch.zeros(2, 4, dtype=i32)
    args = [seq, seq.clone(), seq.clone(), table, ring, pos]
    for i, bad in ((0, torch.zeros(3, dtype=i32)), (1, torch.zeros(2)), (2, torch.zeros(4, dtype=i32)[::2]), (3, torch.zeros(2, 4)), (4, ring.long()), (5, torch.zeros(2, dtype=i32))):
        broken = list(args)
        broken[i] = bad
        with pytest.raises(ValueError):
            binding.cache_plan(*broken, page_size=16, max_tokens=4)
    with pytest.raises(RuntimeError):                      # no CPU fallback
        binding.cache_plan(*args, page_size=16, max_tokens=4)
    bf = torch.bfloat16
    kc, k = torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf)
    slot = torch.zeros(3, dtype=torch.int64)
    for bad in ((k.half(), k, kc, kc, slot), (k, k[:2], kc, kc, slot), (k, k, kc, kc[:, :8], slot), (k, k, kc, kc, slot[:2]), (k, k, kc, kc, slot.int()),
                (k[..., ::2], k[..., ::2], kc[..., ::2], kc[..., ::2], slot), (k.double(), k.double(), kc.double(), kc.double(), slot)):
        with pytest.raises(ValueError):
            binding.cache_append(*bad)
    with pytest.raises(RuntimeError):
        binding.cache_append(k, k, kc, kc, slot)
    q, cu, kv = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    for bad in ((q.half(), kc, kc, table, cu, kv), (q[..., :32], kc, kc, table, cu, kv), (q, kc, kc, table, cu[:2], kv), (q, kc, kc, table, cu, cu),
                (q, kc, kc, table[0], cu, kv), (q.float(), kc.float(), kc.float(), table, cu, kv)):
        with pytest.raises(ValueError):
            binding.chunk_attention(*bad)
    with pytest.raises(RuntimeError):
        binding.chunk_attention(q, kc, kc, table, cu, kv)


def test_binding_refuses_numbers_beyond_32_bits(binding):
    """A descriptor holds 32-bit sizes: a window of 2^32 + 5 must not become one of 5."""
    import torch
    i32, bf = torch.int32, torch.bfloat16
    seq, ring, pos, table = torch.zeros(2, dtype=i32), torch.zeros(8, dtype=i32), torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4, dtype=i32)
    args = [seq, seq.clone(), seq.clone(), table, ring, pos]
    for bad in (dict(page_size=2 ** 32 + 16, max_tokens=4), dict(page_size=-2 ** 32 + 16, max_tokens=4), dict(page_size=16, max_tokens=2 ** 32 + 4),
                dict(page_size=16, max_tokens=-2 ** 32 + 4)):
        with pytest.raises(ValueError):
            binding.cache_plan(*args, **bad)
    wide = torch.zeros(1, dtype=i32).expand(2 ** 31)                 # (no memory behind it: refused before anything is read)
    with pytest.raises(ValueError):
        binding.cache_plan(seq, seq.clone(), seq.clone(), table, wide, pos, page_size=16, max_tokens=4)
    q, kc, cu, kv = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    for window in (2 ** 31, 2 ** 32 + 5, -2 ** 32 + 5):
        with pytest.raises(ValueError):
            binding.chunk_attention(q, kc, kc, table, cu, kv, window=window)
    many = torch.zeros(1, 1, 1, 8, dtype=bf).expand(2 ** 32 + 8, 1, 1, 8)
    with pytest.raises(ValueError):
        binding.chunk_attention(torch.zeros(3, 1, 8, dtype=bf), many, many, table, cu, kv)
    k = torch.zeros(3, 1, 8, dtype=bf)
    with pytest.raises(ValueError):
        binding.cache_append(k, k, many, many, torch.zeros(3, dtype=torch.int64))
    rows = torch.zeros(1, 1, 8, dtype=bf).expand(2 ** 32 + 3, 1, 8)
    with pytest.raises(ValueError):
        binding.chunk_attention(rows, kc[:, :, :1, :8], kc[:, :, :1, :8], table, cu, kv)
    with pytest.raises(ValueError):
        binding.cache_append(rows, rows, kc[:, :, :1, :8], kc[:, :, :1, :8], torch.zeros(1, dtype=torch.int64).expand(2 ** 32 + 3))


def test_binding_refuses_a_stream_of_another_device(binding):
    """The work goes to the tensors' device: a stream of another one could not order it."""
    import types

    import torch
    i32, bf = torch.int32, torch.bfloat16
    seq, ring, pos, table = torch.zeros(2, dtype=i32), torch.zeros(8, dtype=i32), torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4, dtype=i32)
    q, kc, k = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf)
    other = types.SimpleNamespace(device_index=1)
    for call in (lambda: binding.cache_plan(seq, seq, seq, table, ring, pos, page_size=16, max_tokens=4, stream=other),
                 lambda: binding.cache_append(k, k, kc, kc, torch.zeros(3, dtype=torch.int64), stream=other),
                 lambda: binding.chunk_attention(q, kc, kc, table, torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), stream=other)):
        with pytest.raises(ValueError, match="stream"):
            call()


def test_outputs_whose_rows_share_memory_are_refused(binding):
    """A stride of zero on an axis longer than one would let rows of the result, or slots of the cache, overwrite one another."""
    lib = binding.load_library()
    for bad in (dict(o_tok=0), dict(o_head=0)):
        assert lib.specsteer_chunk_attention(_attention(binding, **bad), None) == binding.ERR_INVALID_ARG
    for bad in (dict(kc_page=0), dict(kc_slot=0), dict(kc_head=0), dict(vc_page=0), dict(vc_slot=0), dict(vc_head=0)):
        assert lib.specsteer_cache_append(_append(binding, **bad), None) == binding.ERR_INVALID_ARG
    # the axis of one carries no stride; inputs may be broadcast
    assert lib.specsteer_chunk_attention(_attention(binding, T=0, o_tok=0, q_tok=0, kc_head=0), None) == binding.OK
    assert lib.specsteer_cache_append(_append(binding, T=0, k_tok=0), None) == binding.OK


def test_the_hook_that_stops_loading(binding):
    """Bits 16 to 31 of flags, and what the binding makes of a number of blocks."""
    import torch
    lib = binding.load_library()
    assert lib.specsteer_chunk_attention(_attention(binding, flags=5 << 16, T=0), None) == binding.OK
    assert lib.specsteer_chunk_attention(_attention(binding, flags=5 << 16 | 4, T=0), None) == binding.ERR_INVALID_ARG
    i32, bf = torch.int32, torch.bfloat16
    args = (torch.zeros(3, 4, 64, dtype=bf), torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(8, 16, 2, 64, dtype=bf), torch.zeros(2, 4, dtype=i32),
            torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32))
    for blocks in (-1, 65535, 1 << 40):
        with pytest.raises(ValueError):
            binding.chunk_attention(*args, stop_after=blocks)


def test_attention_sizes_next_to_2_to_the_31(binding):
    """Loops over requests and over tiles of rows step past the last one: what would leave 32 bits is refused, or is the
    generic kernel's, which counts rows in 64 bits."""
    lib, most = binding.load_library(), 2 ** 31 - 1 - 4096
    for bad in (dict(B=most + 1), dict(B=2 ** 31 - 1)):
        assert lib.specsteer_chunk_attention(_attention(binding, **bad), None) == binding.ERR_UNSUPPORTED
        assert lib.specsteer_chunk_attention_workspace(_attention(binding, **bad)) == 0
    assert lib.specsteer_chunk_attention_workspace(_attention(binding, B=most)) > 0
    assert lib.specsteer_chunk_attention_workspace(_attention(binding, T=most)) > 0        # the tensor-core kernel's workspace
    assert lib.specsteer_chunk_attention_workspace(_attention(binding, T=most + 1)) == 0   # the generic kernel needs none
