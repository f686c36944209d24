"""GPU: the bounded waits of the block-scaled products."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def _operands(seed, M, inner, E, N, K):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(M, inner, generator=g, device="cuda", dtype=BF16)
    w = torch.randn(E, N, K, generator=g, device="cuda", dtype=BF16)
    return eat.quant_rows(x) + eat.quant_tiles(w)


@pytest.mark.parametrize("transposed", [False, True])
def test_a_wait_bounds_a_step_and_not_the_call(transposed):
    """A product on SM pairs of several times the limit, none of whose steps takes a hundredth of it."""
    n, limit = 16384, 1_000_000
    xq, xs, wq, ws = _operands(1, n, n, 1, n, n)
    want = eat.block_mm(xq, xs, wq[0], ws[0], transposed=transposed)
    y = torch.full_like(want, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    eat.eat_block_mm_selftest(xq, xs, wq, ws, None, 1, n, n, n, transposed, y, eat.EAT_BF16, limit, status)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) > 2e-6 * limit
    assert status.item() == 0 and torch.equal(y, want)
