"""GPU: the balance loss's exponentials over a wide range of logits."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -23


@pytest.mark.parametrize("T", [50, 900, 5000])
def test_gradient_of_improbable_experts(T):
    """Probabilities down to exp(-60), each with the relative accuracy of fp32.

    Logits are multiples of 1/64, so that their differences are exact.  With 8 experts, in units of 2^-23:
    an exponential 1, a sum of eight 3/2, a quotient 1/2, so 4 for p; dot adds a product and three sums
    (5/2) to that; f - dot, the scale and the products 3 more.  Below 14 of p (f + dot), all of them one
    after the other."""
    from paper_2609_33614_gb300 import build
    build.build()
    E, K = 8, 2
    gen = torch.Generator("cuda").manual_seed(17)
    z = torch.round(-60.0 * torch.rand(T, E, generator=gen, device="cuda") * 64) / 64
    z[:, 0] = 0.0
    # (the probable expert is not selected: f - dot is as large as f + dot, and p's error shows whole)
    idx = torch.randint(1, E, (T, K), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.full((1,), 0.75, device="cuda")
    loss, counts, n = eat.balance_loss(z, idx)
    d = eat.balance_grad(z, counts, n, g).double()
    p = torch.softmax(z.double(), 1)
    f = counts.double() / counts.sum()
    dot = (p * f).sum(1, keepdim=True)
    scale = 0.75 * E / T
    assert ((d - scale * p * (f - dot)).abs() <= 14 * U32 * scale * p * (f + dot)).all()
    # (sums over the tokens as well)
    want = float(E * (p.mean(0) * f).sum())
    assert abs(float(loss) - want) <= 64 * U32 * want
