"""GPU: the gated activation over the gates' whole range, against 64 bits.

Tolerances, in units of 2^-24 of the result.  CUDA's tables: expf 2 units in the last place (4 of these), __expf
2 + |1.173 x| (twice as many of these), rcp.approx 1 (2); a product, a sum or a rounded reciprocal 1.
Subnormal numbers lie 2^-149 apart in fp32 and 2^-133 in bf16 (7 bits behind 2^-126): a rounding there is off
by half of that.
"""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
U32, U16 = 2.0 ** -24, 2.0 ** -8


def _inputs(dtype, F, scale):
    gen = torch.Generator("cuda").manual_seed(int(scale) % 97)
    edges = torch.tensor([-100.0, -89.0, -88.8, -88.5, -87.5, -64.5, -64.0, -63.9, -1.28, -1e-3, 0.0, 1e-3, 17.0,
                          64.0, 88.8, 100.0], device="cuda")
    gate = torch.cat([edges, torch.linspace(-100, 100, 3 * F - 16, device="cuda")]).view(3, F)
    up = scale * (0.5 + torch.rand(3, F, generator=gen, device="cuda"))
    up *= torch.where(torch.rand(3, F, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    return gate.to(dtype), up.to(dtype)


def _units(dtype, gate):
    """Of a sigmoid: its exponential, the sum and the reciprocal; far below 0 two roots of the exponential, each of
    half the argument."""
    x = gate.double().abs()
    if dtype == F32:
        return 8.0 + 0 * x  # 4 + 1 + 1, or 2 * 4
    return 8.0 + 2.346 * x  # 2 (2 + 1.173 x) + 1 + 2, or 2 * 2 (2 + 0.587 x)


def _bound(dtype):
    return U32 if dtype == F32 else U16


def _least(dtype):
    return 2.0 ** -148 if dtype == F32 else 2.0 ** -148 + 2.0 ** -134


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("F", [1024, 1001])
@pytest.mark.parametrize("scale", [1.0, 1e10, 1e30])
def test_values(dtype, F, scale):
    gate, up = _inputs(dtype, F, scale)
    h = eat.swiglu(torch.cat([gate, up], 1)).double()
    g, u = gate.double(), up.double()
    want = g * torch.sigmoid(g) * u
    tol = (_units(dtype, gate) + 3) * U32 + _bound(dtype)
    assert ((h - want).abs() <= tol * want.abs() + _least(dtype)).all()
    at = (gate < -88.7) & (want.abs() > 1e-37)
    assert at.any() and (h[at] != 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("F", [1024, 1001])
@pytest.mark.parametrize("scale", [1.0, 1e10, 1e30])
def test_gradients(dtype, F, scale):
    gate, up = _inputs(dtype, F, scale)
    dh = _inputs(dtype, F, 1.0)[1]
    d = eat.swiglu_grad(torch.cat([gate, up], 1), dh).double()
    g, u, dd = gate.double(), up.double(), dh.double()
    s = torch.sigmoid(g)
    want = torch.cat([dd * u * s * (1 + g * torch.sigmoid(-g)), dd * g * s], 1)
    # 1 + g (1 - s): the magnitudes of what is added, s as far off in 1 - s as it is itself
    inner = 1 + g.abs() * torch.sigmoid(-g)
    units = _units(dtype, gate)
    first = (dd * u * s).abs() * (inner * (units + 6) + g.abs() * s * (units + 1))
    mag = torch.cat([first, (dd * g * s).abs() * (units + 3)], 1) * U32
    least = 2 * (1 + g.abs().max()) * 2.0 ** -148 + _least(dtype)
    assert ((d - want).abs() <= mag + _bound(dtype) * want.abs() + least).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("F", [1024, 1001])
def test_e4m3_blocks_of_far_gates(dtype, F):
    """Blocks whose gates are all far below 0, and large ups: their largest magnitude is no longer 0."""
    gate, up = _inputs(dtype, F, 1e10)
    gate = torch.linspace(-92, -89, 3 * F, device="cuda").view(3, F).to(dtype)
    q, scale = eat.swiglu_fp8(torch.cat([gate, up], 1))
    g, u = gate.double(), up.double()
    want = g * torch.sigmoid(g) * u
    s = scale.double().t().repeat_interleave(128, 1)[:, :F]
    assert (s != 1).all()
    t = want / s
    step = torch.maximum(t.abs() * 2.0 ** -4, torch.full_like(t, 2.0 ** -10))
    # (e4m3 of fp32 rows takes bf16's exponential too)
    assert ((q.double() - t).abs() <= step + (_units(BF16, gate) + 6) * U32 * t.abs()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("F", [1024, 1001])
def test_far_gates_leave_their_neighbours_alone(dtype, F):
    """Bits of an element do not depend on the gates beside it, nor on where the rows begin."""
    gate, up = _inputs(dtype, F, 1.0)
    gate = (gate.float() / 2).to(dtype)  # none below -64
    dh = _inputs(dtype, F, 1.0)[1]
    mixed = gate.clone()
    mixed[:, ::5] = -80.0
    near = torch.ones(F, dtype=torch.bool, device="cuda")
    near[::5] = False
    h, want = eat.swiglu(torch.cat([mixed, up], 1)), eat.swiglu(torch.cat([gate, up], 1))
    d, dwant = eat.swiglu_grad(torch.cat([mixed, up], 1), dh), eat.swiglu_grad(torch.cat([gate, up], 1), dh)
    assert torch.equal(h[:, near], want[:, near])
    assert torch.equal(d[:, near.repeat(2)], dwant[:, near.repeat(2)])
    buf = torch.zeros(3 * 2 * F + 8, dtype=dtype, device="cuda")
    moved = buf[1:1 + 6 * F].view(3, 2 * F)
    moved.copy_(torch.cat([mixed, up], 1))
    assert torch.equal(eat.swiglu(moved), h) and torch.equal(eat.swiglu_grad(moved, dh), d)
