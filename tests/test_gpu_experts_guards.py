"""GPU: the experts' calls write their outputs and nothing beside them, whatever offsets and slots hold; and the
weights' gradient of rows whose offsets pass 32 bits."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
CODE = {BF16: eat.EAT_BF16, F32: eat.EAT_F32}
PAD = 1024  # elements on either side


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def _randn(seed, *shape, dtype=BF16):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


class Guards:
    """Outputs between bands of bytes that no call may touch."""

    def __init__(self):
        self.bufs = []

    def out(self, dtype, *shape, off=0):
        n = 1
        for s in shape:
            n *= s
        size = torch.empty((), dtype=dtype).element_size()
        buf = torch.full(((n + 2 * PAD) * size,), 0x55, dtype=torch.uint8, device="cuda")
        lo = (PAD + off) * size
        self.bufs.append((buf, lo, lo + n * size))
        return buf[lo:lo + n * size].view(dtype).view(shape)

    def check(self):
        torch.cuda.synchronize()
        for buf, lo, hi in self.bufs:
            assert (buf[:lo] == 0x55).all() and (buf[hi:] == 0x55).all()


def _bad(kind, T, K, E, seed=9):
    """(offsets, slot) that no sort makes."""
    M, top = T * K, 2 ** 31 - 1
    g = torch.Generator("cuda").manual_seed(seed)
    slot = torch.randint(-M, 2 * M, (T, K), generator=g, device="cuda").to(torch.int32)
    offsets = torch.randint(-M, 2 * M, (E + 1,), generator=g, device="cuda").to(torch.int32)
    if kind == "ends":
        slot[0::3], slot[1::3] = top, -top - 1
        offsets[0::2], offsets[1::2] = top, -top - 1
    if kind == "edges":
        slot[:] = M
        slot[::2] = M - 1
        offsets[:] = M + 1
        offsets[::2] = 0
    return offsets, slot


@pytest.mark.parametrize("kind", ["random", "ends", "edges"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,K,E,d,off", [(1, 1, 1, 1, 0), (33, 3, 5, 136, 0), (70, 8, 64, 1001, 3), (300, 2, 7, 2048, 0)])
def test_rows_of_slots_that_no_sort_makes(T, K, E, d, off, dtype, kind):
    offsets, slot = _bad(kind, T, K, E)
    M, c, G = T * K, CODE[dtype], Guards()
    x, dy, rows = _randn(1, T, d, dtype=dtype), _randn(2, T, d, dtype=dtype), _randn(3, M, d, dtype=dtype)
    w = torch.rand(T, K, generator=torch.Generator("cuda").manual_seed(4), device="cuda")
    eat.eat_expert_gather(x, T, K, E, d, c, slot, offsets, G.out(dtype, M, d, off=off), c, None)
    eat.eat_expert_gather(x, T, K, E, d, c, slot, offsets, G.out(E4M3, M, d, off=off), eat.EAT_FP8_E4M3,
                          G.out(F32, -(-d // 128), M))
    for weight in (w, None):
        y = G.out(dtype, T, d, off=off)
        eat.eat_expert_combine(rows, T, K, d, c, slot, weight, y)
        used = (slot >= 0) & (slot < M)  # the sum takes the slots that are rows
        f = torch.where(used, w.double() if weight is not None else 1.0, 0.0)
        terms = f[..., None] * rows.double()[slot.clamp(0, M - 1).long()]
        want, mag = terms.sum(1), terms.abs().sum(1)
        u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
        assert ((y.double() - want).abs() <= u * want.abs() + 2 * K * 2.0 ** -24 * mag).all()
    dw = G.out(F32, T, K)
    eat.eat_expert_combine_grad(dy, rows, T, K, E, d, c, slot, offsets, w, G.out(dtype, M, d, off=off), dw)
    assert (dw[~used] == 0).all()
    G.check()


@pytest.mark.parametrize("kind", ["random", "ends", "edges"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,E,off", [(1, 1, 1, 0), (96, 128, 4, 0), (700, 136, 64, 0), (500, 1001, 7, 1)])
def test_columns_of_offsets_that_no_sort_makes(M, K, E, off, dtype, kind):
    offsets, _ = _bad(kind, M, 1, E)
    x, c, G = _randn(5, M, K, dtype=dtype), CODE[dtype], Guards()
    rows, blocks = eat.eat_quant_columns_rows(M, E), eat.eat_quant_columns_blocks(M, E)
    for q, scale in ((None, None), (G.out(E4M3, M, K, off=off), G.out(F32, -(-K // 128), M))):
        eat.eat_quant_columns(x, M, K, c, offsets, E, q, scale, G.out(E4M3, rows, K, off=off),
                              G.out(F32, blocks, K))
    G.check()


@pytest.mark.parametrize("kind", ["random", "ends", "edges"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,E,cols,inner", [
    (96, 4, 64, 128), (40, 4, 8192, 144), (160, 4, 8192, 144), (400, 4, 8192, 272), (500, 2, 8192, 272),
    (2000, 4, 4096, 128), (2000, 4, 4080, 1680)])
def test_products_of_offsets_that_no_sort_makes(M, E, cols, inner, transposed, dtype, kind):
    """Every height of tile, and SM pairs (2000 rows)."""
    offsets, _ = _bad(kind, M, 1, E)
    N, K = (inner, cols) if transposed else (cols, inner)
    (xq, xs), (wq, ws) = eat.quant_rows(_randn(6, M, inner)), eat.quant_tiles(_randn(7, E, N, K))
    G = Guards()
    eat.eat_block_mm(xq, xs, wq, ws, offsets, E, M, N, K, transposed, G.out(dtype, M, cols), CODE[dtype])
    if cols <= 4096:
        g, x = _randn(8, M, 64), _randn(9, M, 144)
        sorted_ = (torch.arange(E + 1, device="cuda") * M // E).to(torch.int32)
        (gq, gs), (cq, cs) = eat.quant_columns(g, sorted_), eat.quant_columns(x, sorted_)
        eat.eat_block_mm_grad(gq, gs, cq, cs, offsets, E, len(gq), len(gs), 64, 144, G.out(dtype, E, 64, 144),
                              CODE[dtype])
    G.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,K,E,d,off", [(1, 1, 1, 1, 0), (33, 3, 5, 136, 0), (70, 8, 64, 1001, 3), (2049, 8, 60, 128, 0)])
def test_outputs_of_a_sorted_step(T, K, E, d, off, dtype):
    """The calls as they follow each other: every output whole, nothing beside it."""
    c, G = CODE[dtype], Guards()
    idx = torch.randint(-1, E + 1, (T, K), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.int32)
    M = T * K
    offsets, slot = G.out(torch.int32, E + 1), G.out(torch.int32, T, K)
    work = torch.empty(max(16, eat.eat_expert_sort_workspace(T, K, E)), dtype=torch.uint8, device="cuda")
    eat.eat_expert_sort(idx, T, K, E, None, offsets, slot, work)
    x = _randn(2, T, d, dtype=dtype)
    rows = G.out(dtype, M, d, off=off)
    eat.eat_expert_gather(x, T, K, E, d, c, slot, offsets, rows, c, None)
    assert torch.equal(rows, eat.expert_gather(x, slot, offsets))
    q, scale = G.out(E4M3, M, d, off=off), G.out(F32, -(-d // 128), M)
    eat.eat_quant_rows(rows, M, d, c, q, scale)
    want = eat.quant_rows(rows.clone())
    assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(scale, want[1])
    tq, ts = G.out(E4M3, M, d, off=off), G.out(F32, -(-M // 128), -(-d // 128))
    eat.eat_quant_tiles(rows, 1, M, d, c, tq, ts)
    gu, dh = _randn(3, T, 2 * d, dtype=dtype), _randn(4, T, d, dtype=dtype)
    eat.eat_swiglu(gu, T, d, c, G.out(dtype, T, d, off=off), c)
    eat.eat_swiglu(gu, T, d, c, G.out(E4M3, T, d, off=off), eat.EAT_FP8_E4M3, G.out(F32, -(-d // 128), T))
    eat.eat_swiglu_grad(gu, dh, T, d, c, G.out(dtype, T, 2 * d, off=off))
    G.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_gradient_of_an_expert_that_is_not_all_there(dtype):
    """Offsets of more rows than the operands have: NaN, where zeros would pass for a gradient."""
    g, x = _randn(1, 100, 48), _randn(2, 100, 272)
    made = torch.tensor([0, 60, 60, 100], device="cuda", dtype=torch.int32)
    (gq, gs), (xq, xs) = eat.quant_columns(g, made), eat.quant_columns(x, made)
    want = eat.block_mm_grad(gq, gs, xq, xs, offsets=made, dtype=dtype)
    assert want.isfinite().all() and (want[1] == 0).all()
    for other, whole in (([0, 60, 60, 400], 2), ([0, 60, 2000, 2000], 1)):
        dw = eat.block_mm_grad(gq, gs, xq, xs, offsets=torch.tensor(other, device="cuda", dtype=torch.int32), dtype=dtype)
        assert torch.equal(dw[:whole], want[:whole]) and dw[whole].isnan().all()
        assert (dw[whole + 1:] == 0).all()  # (without rows)


def test_weights_gradient_of_rows_far_into_a_buffer():
    """The last block of rows, whose bytes begin beyond 2^32, is all that g is not 0 in."""
    T, d, N, n = 70000, 65536, 16, 112
    x = torch.empty(T, d, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    g = torch.zeros(T, N, dtype=BF16, device="cuda")
    g[-n:] = _randn(2, n, N)
    (gq, gs), (xq, xs) = eat.quant_columns(g), eat.quant_columns(x)
    assert T % 128 == n and (T - n) * d > 2 ** 32
    dw = eat.block_mm_grad(gq, gs, xq, xs, dtype=F32)
    u, v = gq[T - n:].double() * gs[-1].double(), xq[T - n:].double() * xs[-1].double()
    assert v[n:].abs().sum() == 0  # (what pads)
    want, mag = u.t() @ v, u.abs().t() @ v.abs()
    # a block of 128 on the tensor cores, and two products of scales; the other blocks add zeros
    assert ((dw.double() - want).abs() <= 2.0 ** -24 * want.abs() + 12 * 2.0 ** -23 * mag).all()
    assert want.abs().max() > 1
