"""GPU: vocabulary rows whose logits are infinite, in the head's loss and gradient.

Tolerances as for finite logits: bf16 roundings of P, of one more factor and of the result (u16 each, of
the sum of magnitudes), and a logit's own error of (d / 16 + 2) 2^-23 sum |x w|.
"""
import math

import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def _case(T, V, d, seed):
    """x[:, 0] is positive: a vocabulary row with an infinite first element has an infinite logit."""
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(T, d, generator=gen, device="cuda")
    x[:, 0] = x[:, 0].abs() + 0.5
    w = 0.1 * torch.randn(V, d, generator=gen, device="cuda")
    y = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    g = (0.5 + torch.rand(T, generator=gen, device="cuda")) / T
    return x.bfloat16(), w.bfloat16(), y, g


@pytest.mark.parametrize("V", [900, 5003])
@pytest.mark.parametrize("T", [1, 5, 64, 100, 129, 300])
def test_gradient_with_rows_without_probability(T, V):
    """Vocabulary rows of logit -inf: dw is 0 there, except that of one token's target."""
    d = 128
    x, w, y, g = _case(T, V, d, 5)
    dead = torch.zeros(V, dtype=torch.bool, device="cuda")
    dead[100:2 * V // 3:3] = True
    dead[V - 1] = True
    w[dead, 0] = -math.inf
    y = torch.where(dead[y.long()], y % 100, y)
    lost = T > 1
    if lost:
        y[1] = 100  # a dead row
    nll, lse, dx, dw = eat.EatHead(w, T, grad=True).nll_grad(x, y, g)
    x64, w64, g64 = x.double(), w.double(), g.double()
    logits = x64 @ torch.where(dead[:, None], 0.0, w64).T
    logits[:, dead] = -math.inf
    z = torch.logsumexp(logits, 1)
    rows = torch.arange(T, device="cuda")
    want = z - logits[rows, y.long()]
    dl = (d / 16 + 2) * U32 * float((x64.abs() @ w64[~dead].abs().T).max()) + 64 * U32
    assert ((lse.double() - z).abs() <= 2 * dl).all()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    if lost:
        assert float(nll[1]) == math.inf
        keep[1] = False
    assert ((nll.double() - want).abs() <= 2 * dl)[keep].all()
    p = torch.softmax(logits, 1)
    p[rows, y.long()] -= 1.0
    p *= g64[:, None]
    k = 2 * U16 + 4 * dl
    ref, mag = p.T @ x64, p.abs().T @ x64.abs()
    assert ((dw.double() - ref).abs() <= 1.01 * k * mag + U16 * ref.abs() + 1e-30).all()
    clean = dead.clone()
    if lost:
        clean[100] = False
    assert (dw[clean] == 0).all()
    # (column 0 of w holds -inf, and 0 times that is NaN)
    ref, mag = p @ w64[:, 1:], p.abs() @ w64[:, 1:].abs()
    assert ((dx[:, 1:].double() - ref).abs() <= 1.01 * k * mag + U16 * ref.abs() + 1e-30).all()


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("V", [900, 20000])
@pytest.mark.parametrize("T", [2, 20, 50, 100, 300])
def test_a_logit_of_plus_infinity_costs_infinitely_much(T, V, grad):
    """nll and lse of a token with a logit of +inf beside its target's are inf; the others', for whom
    the row's logit is -inf, are those of the other rows."""
    d, row = 128, V // 2
    x, w, y, g = _case(T, V, d, 7)
    x[::2, 0] = -x[::2, 0]
    w[row, 0] = math.inf
    y = torch.where(y == row, row + 1, y)
    head = eat.EatHead(w, T, grad=grad)
    nll, lse = head.nll_grad(x, y, g)[:2] if grad else head.nll(x, y)
    assert (nll[1::2] == math.inf).all() and (lse[1::2] == math.inf).all()
    x64, w64 = x[::2].double(), w.double()
    w64[row] = 0.0
    logits = x64 @ w64.T
    logits[:, row] = -math.inf
    z = torch.logsumexp(logits, 1)
    want = z - logits.gather(1, y[::2, None].long())[:, 0]
    dl = (d / 16 + 2) * U32 * float((x64.abs() @ w64.abs().T).max()) + 64 * U32
    assert ((lse[::2].double() - z).abs() <= 2 * dl).all()
    assert ((nll[::2].double() - want).abs() <= 2 * dl).all()
