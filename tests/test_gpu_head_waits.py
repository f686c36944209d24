"""GPU: the head's bounded waits are each for a step of a call, whose whole time they do not bound."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu


def test_a_call_may_take_longer_than_the_limit_of_its_waits():
    """Calls of several times the limit, none of whose steps (a tile's sums: at most 512 k-blocks) takes a
    quarter of it."""
    from paper_2609_33614_gb300 import build
    build.build()
    T, V, d, limit = 32768, 32768, 4096, 1_000_000
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(T, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = 0.02 * torch.randn(V, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    n = 8192  # one piece of the gradient
    g = torch.full((n,), 1.0 / n, device="cuda")
    head = eat.EatHead(w, T, grad=True)
    want = head.nll(x, y) + head.nll_grad(x[:n], y[:n], g)
    begin, mid, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    eat.eat_head_selftest_wait_limit(head.h, limit)
    begin.record()
    got = head.nll(x, y)
    mid.record()
    got += head.nll_grad(x[:n], y[:n], g)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(mid) > 2e-6 * limit and mid.elapsed_time(end) > 2e-6 * limit
    for a, b in zip(got, want):
        assert torch.equal(a, b) and a.isfinite().all()
    eat.eat_head_selftest_wait_limit(head.h, 0)
    assert torch.equal(head.nll(x, y)[0], want[0])  # (the handle has not failed)
    head.close()


def test_limits_out_of_range_are_refused():
    w = torch.zeros(64, 64, device="cuda", dtype=torch.bfloat16)
    head = eat.EatHead(w, 4)
    for limit in (-1, 999_999, 10 ** 9 + 1):
        with pytest.raises(eat.EatError, match="limit_ns"):
            eat.eat_head_selftest_wait_limit(head.h, limit)
    head.close()
