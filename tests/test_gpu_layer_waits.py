"""GPU: the expert kernels' bounded waits are each for a step of a call, whose whole time they do not bound."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("fp8,shared", [(False, 0), (False, 2), (True, 0)])
def test_a_call_may_take_longer_than_the_limit_of_its_waits(fp8, shared):
    """Launches of several times the limit, none of whose steps (a tile's sums: at most 224 k-blocks of 64)
    takes a fifth of it."""
    E, F, d, T, limit = 8, 14336, 4096, 32768, 1_000_000
    gen = torch.Generator("cuda").manual_seed(7)
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(0.02).to(dtype)
    scales = {}
    if fp8:
        ones = lambda *s: torch.ones(*s, device="cuda")
        scales = dict(w_gate_scale=ones(E, F), w_up_scale=ones(E, F), w_down_scale=ones(E, d))
    more = dict(ws_gate=make(shared, F, d), ws_up=make(shared, F, d), ws_down=make(shared, d, F)) if shared else {}
    router = torch.randn(E, d, generator=gen, device="cuda").mul_(0.02)
    layer = eat.EatLayer(router, torch.zeros(E, device="cuda"), make(E, F, d), make(E, F, d), make(E, d, F), T,
                         eat.eat_default_params(2), scales=scales, **more)
    x = torch.randn(T, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    accounts = [t.clone() for t in layer.accounts()]
    want = layer.forward(x)
    layer.set_accounts(*accounts)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    eat.eat_selftest_wait_limit(layer.h, limit)
    begin.record()
    got = layer.forward(x)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) > 5e-6 * limit
    assert eat.eat_get_counters(layer.h)["status"] == 0
    assert torch.equal(got, want) and got.isfinite().all()
    for bad in (-1, 999_999, 10 ** 9 + 1):
        with pytest.raises(eat.EatError, match="limit_ns"):
            eat.eat_selftest_wait_limit(layer.h, bad)
    eat.eat_selftest_wait_limit(layer.h, 0)
    layer.close()
