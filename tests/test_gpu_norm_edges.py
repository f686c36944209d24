"""GPU: the RMS norm at the ends of fp32's range."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -23
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("d,off", [(64, 0), (100, 0), (1024, 0), (4096, 0), (1024, 1)])
def test_e4m3_rows_of_tiny_values(d, off, residual, dtype):
    """Rows whose largest product h gamma lies between 2^-100 and 2^-126, zeros among them: scaled by
    max / 448 as any others; below 1e-35 (after the norm) the scale is 1 and the bytes are 0.

    Products near 2^-126 are rounded to multiples of 2^-149, 2^-23 of the row's largest; so are, of
    themselves, the row's factors.  In units of the scale (largest 448) that is below 448 x 2^-20, beside
    half a step of e4m3 (2^-4 of a value, 2^-10 at least)."""
    tops = [-100, -110, -117, -118, -119, -120, -121, -123, -125, -126, -127, -140, None]
    T = len(tops)
    gen = torch.Generator("cuda").manual_seed(3)
    u = torch.rand(T, d, generator=gen, device="cuda", dtype=torch.float64) - 0.5
    gamma = 0.9 + 0.2 * torch.rand(d, generator=gen, device="cuda")
    u[:, ::5] = 0.0
    u[:, 3], gamma[3] = -1.0, 1.0
    for t, e in enumerate(tops):
        u[t] *= 0.0 if e is None else 2.0 ** e
    buf = torch.zeros(T * d + 8, dtype=dtype, device="cuda")
    x = buf[off:off + T * d].view(T, d)
    x.copy_(u.to(dtype))
    r = torch.zeros_like(x) if residual else None
    q, scale, h = eat.rms_norm_fp8(x, gamma, EPS, residual=r)
    assert torch.equal(h, x)
    s = x.double()
    want = s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * gamma.double()
    top = want.abs().amax(1)
    scaled = top > 1e-35
    assert scaled.sum() == 10 and ((top - 1e-35).abs() > 1e-37).all()
    assert (scale[~scaled] == 1.0).all() and (q[~scaled].float() == 0).all()
    ref = top[scaled] / 448.0
    assert ((scale[scaled].double() - ref).abs() <= 16 * U32 * ref).all()
    v, got = want[scaled] / ref[:, None], q[scaled].double()
    assert (got[v == 0] == 0).all()
    step = torch.maximum(v.abs() * 2.0 ** -4, torch.full_like(v, 2.0 ** -10))
    assert ((got - v).abs() <= step * (1 + 1e-5) + 448 * 2.0 ** -20).all()
