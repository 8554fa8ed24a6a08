"""A round over trees of drafts on the GPU: arguments at the ends of what the operators accept."""
import ctypes as C

import pytest
import torch

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
