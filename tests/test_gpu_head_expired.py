"""GPU: every output of a head's call whose wait gave up."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [5, 60, 127, 300])
def test_gradients_of_an_expired_call_are_nan(T):
    """dw is NaN in every entry (an update with it would not go unseen), dx in the counted rows and 0 in
    the ignored ones."""
    from paper_2609_33614_gb300 import build
    build.build()
    V, d = 700, 128
    gen = torch.Generator("cuda").manual_seed(9)
    x = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    w = (0.05 * torch.randn(V, d, generator=gen, device="cuda")).bfloat16()
    y = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    y[2] = -1
    head = eat.EatHead(w, T, grad=True)
    eat.eat_head_selftest_expire_wait(head.h, 10_000)
    nll, lse, dx, dw = head.nll_grad(x, y, torch.ones(T, device="cuda"))
    torch.cuda.synchronize()
    on = y >= 0
    assert nll[on].isnan().all() and lse[on].isnan().all() and dx[on].isnan().all()
    assert dw.isnan().all()
    assert (nll[~on] == 0).all() and (dx[~on] == 0).all()
    head.close()
