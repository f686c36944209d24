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


LIMIT = 1_000_000  # the copies of a step take a thousandth of it


def _guarded(shape, dtype):
    """A tensor of 7s between two others."""
    n, pad = shape.numel(), 4096
    buf = torch.full((n + 2 * pad,), 7.0, dtype=dtype, device="cuda")
    return buf[pad:pad + n].view(shape), (buf[:pad], buf[pad + n:])


def _check(got, guards, want, dead, status):
    """NaN exactly where a tile was not finished, the call's results elsewhere."""
    assert status.item() != 0 and status.item() & ~(1 | 2 | 4 | 8 | 16 | 32 | 64) == 0
    assert all((g == 7).all() for g in guards)
    assert dead.any() and not dead.all()
    assert got[dead].isnan().all()
    assert torch.equal(got[~dead], want[~dead])


def _ctas(pairs):
    n = torch.cuda.get_device_properties(0).multi_processor_count
    return n // 2 if pairs else n


# rows, columns of the output, sums, its tiles' columns: every height of tile, and SM pairs; with
# 400 columns of tiles a CTA has several
SHAPES = [(8, 128 * 400, 528, 128), (40, 128 * 400, 400, 128), (64, 128 * 400, 640, 128), (256, 128 * 100, 272, 128),
          (256, 256 * 200, 528, 256), (200, 256 * 200 - 112, 400, 256), (300, 256 * 100, 1680, 256)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("done", ["nothing", "a part of a tile", "one tile"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("rank", [0, 1])
def test_an_expired_wait_leaves_nan_in_the_tiles_that_are_not_done(shape, rank, done, transposed, dtype):
    """Copies that end on the host's word: the call returns, with a status, and the next one is right."""
    M, cols, inner, width = shape
    pairs = width == 256
    N, K = (inner, cols) if transposed else (cols, inner)
    xq, xs, wq, ws = _operands(2, M, inner, 1, N, K)
    want = eat.block_mm(xq, xs, wq[0], ws[0], transposed=transposed, dtype=dtype)
    y, guards = _guarded(want.shape, dtype)
    nkb = -(-inner // 128)
    copies = {"nothing": 0, "a part of a tile": nkb - 1, "one tile": nkb}[done]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eat.eat_block_mm_selftest(xq, xs, wq, ws, None, 1, M, N, K, transposed, y,
                              eat.EAT_BF16 if dtype == BF16 else eat.EAT_F32, LIMIT, status, cta=rank,
                              copies=copies)
    torch.cuda.synchronize()
    # tiles go (columns, rows): those of CTA `rank`, or of the first pair
    high = -(-M // (256 if M > 128 else 128))
    count, step = -(-cols // width) * high, _ctas(pairs)
    first = 0 if pairs else rank
    height = -(-(-(-M // high)) // 16) * 16
    dead = torch.zeros(M, cols, dtype=torch.bool, device="cuda")
    for i, u in enumerate(range(first, count, step)):
        if i >= copies // nkb:
            r, c = u % high * height, u // high * width
            dead[r:r + height, c:c + width] = True
    if not dead.any():  # (all of the CTA's tiles were done)
        assert status.item() == 0 and torch.equal(y, want)
        return
    _check(y, guards, want, dead, status)
    again = eat.block_mm(xq, xs, wq[0], ws[0], transposed=transposed, dtype=dtype)
    assert torch.equal(again, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("done", ["nothing", "a part of a tile", "one tile"])
@pytest.mark.parametrize("N,K", [(256, 128 * 400), (512, 128 * 200), (272, 144)])
@pytest.mark.parametrize("cta", [0, 2])
def test_an_expired_wait_of_the_weights_gradient(N, K, cta, done, dtype):
    R = 300
    gen = torch.Generator("cuda").manual_seed(4)
    g, x = (torch.randn(R, n, generator=gen, device="cuda", dtype=BF16) for n in (N, K))
    (gq, gs), (xq, xs) = eat.quant_columns(g), eat.quant_columns(x)
    want = eat.block_mm_grad(gq, gs, xq, xs, dtype=dtype)
    dw, guards = _guarded(want.shape, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    copies = {"nothing": 0, "a part of a tile": 2, "one tile": 3}[done]
    eat.eat_block_mm_grad_selftest(gq, gs, xq, xs, None, 1, len(gq), len(gs), N, K, dw,
                                   eat.EAT_BF16 if dtype == BF16 else eat.EAT_F32, LIMIT, status, cta=cta,
                                   copies=copies)
    torch.cuda.synchronize()
    high = -(-N // 256)
    height = -(-(-(-N // high)) // 16) * 16
    dead = torch.zeros(N, K, dtype=torch.bool, device="cuda")
    for i, u in enumerate(range(cta, -(-K // 128) * high, _ctas(False))):
        if i >= copies // 3:
            r, c = u % high * height, u // high * 128
            dead[r:r + height, c:c + 128] = True
    if not dead.any():
        assert status.item() == 0 and torch.equal(dw, want)
        return
    _check(dw, guards, want, dead, status)
    assert torch.equal(eat.block_mm_grad(gq, gs, xq, xs, dtype=dtype), want)


@pytest.mark.parametrize("split,N", [([200, 0, 300, 17], 2048), ([5, 0, 9, 3], 2048), ([400] * 8, 4096)])
def test_rows_behind_the_last_expert_are_zeros_all_the_same(split, N):
    E, R, K = len(split), sum(split), 400
    M = R + 700
    xq, xs, wq, ws = _operands(5, M, K, E, N, K)
    offsets = torch.tensor([0] + split, device="cuda").cumsum(0).to(torch.int32)
    want = eat.block_mm(xq, xs, wq, ws, offsets=offsets)
    y, guards = _guarded(want.shape, BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eat.eat_block_mm_selftest(xq, xs, wq, ws, offsets, E, M, N, K, False, y, eat.EAT_BF16, LIMIT, status,
                              cta=0, copies=1)
    torch.cuda.synchronize()
    assert status.item() != 0 and all((g == 7).all() for g in guards)
    assert (y[R:] == 0).all()
    dead = y.isnan()
    assert dead.any() and torch.equal(y[~dead], want[~dead])
    assert dead[0, :128].all() and not dead.all(1).any()
