"""GPU: the gated activation's gradient written over its rows."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,F,off", [(1, 1, 0), (3, 7, 0), (40, 129, 1), (33, 1001, 3), (300, 721, 0), (33, 200, 0),
                                     (17, 4096, 0), (2, 65536, 0), (9, 65535, 1)])
def test_as_into_another_tensor(R, F, off, dtype):
    gen = torch.Generator("cuda").manual_seed(R + F)
    gu = (4 * torch.randn(R, 2 * F, generator=gen, device="cuda")).to(dtype)
    gu[0, 0] = -80.0
    dh = torch.randn(R, F, generator=gen, device="cuda").to(dtype)
    buf = torch.full((gu.numel() + 64,), 7.0, dtype=dtype, device="cuda")
    own = buf[16 + off:16 + off + gu.numel()].view_as(gu)
    own.copy_(gu)
    want = eat.swiglu_grad(gu, dh)
    eat.eat_swiglu_grad(own, dh, R, F, eat.EAT_F32 if dtype == torch.float32 else eat.EAT_BF16, own)
    assert torch.equal(own, want)
    assert (buf[:16 + off] == 7).all() and (buf[16 + off + gu.numel():] == 7).all()
