"""A round over trees of drafts on the GPU: arguments at the ends of what the operators accept."""
import ctypes as C

import pytest
import torch

import _tree

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def binding():
    from paper_2603_16219_b200 import binding, build
    build.build()
    return binding


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
