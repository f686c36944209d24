"""GPU: tokens sorted by expert and back, e4m3 with a scale for each block of 128 and its products, and the
gated activation, with their gradients, against plain 64-bit implementations.

Tolerances.  A rounding to bf16 moves a value by at most U16 = 2^-8 of itself, to fp32 by 2^-24, to
e4m3 by 2^-4 (below 2^-6 of its scale: by 2^-10).  A sum of n terms in fp32 is off by at most n 2^-24 of the
sum of magnitudes; a block of 128 on the tensor cores by (128 / 16 + 2) 2^-23 of it, as they truncate.
"""
import math

import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24
BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(*shape, generator=_gen(seed), device="cuda")


def _offset(t, n):
    """The same values n elements into a larger buffer (another alignment)."""
    buf = torch.zeros(t.numel() + 64, dtype=torch.uint8 if t.dtype == E4M3 else t.dtype, device="cuda")
    v = buf[n:n + t.numel()].view(t.dtype).view(t.shape)
    v.copy_(t)
    return v


def _u(dtype):
    return U16 if dtype == BF16 else U32


def _idx(seed, T, E, K):
    """Selections: mostly experts, some -1 and some beyond E, now and then the same one twice."""
    g = _gen(seed)
    idx = torch.randint(0, E, (T, K), generator=g, device="cuda")
    idx = torch.where(torch.rand(T, K, generator=g, device="cuda") < 0.3, -1, idx)
    if T > 3:
        idx[1] = -1
        idx[2] = E
        idx[3] = 0
    return idx.to(torch.int32)


def _sorted(idx, E, mask=None):
    """(offsets, slot, entry of each row) in plain torch."""
    flat = idx.flatten().cpu().long()
    if mask is not None:
        flat = torch.where(mask.cpu().bool().repeat_interleave(idx.shape[1]), flat, -1)
    entries = [(flat == e).nonzero()[:, 0] for e in range(E)]
    offsets = torch.tensor([0] + [len(v) for v in entries]).cumsum(0)
    entry = torch.cat(entries)
    slot = torch.full_like(flat, -1)
    slot[entry] = torch.arange(len(entry))
    return (offsets.to(torch.int32).cuda(), slot.view(idx.shape).to(torch.int32).cuda(),
            entry.cuda())


SIZES = [(1, 1, 1), (1, 64, 8), (2, 3, 16), (5, 256, 2), (300, 8, 2), (1024, 60, 8), (1025, 64, 8),
         (9001, 200, 5), (40000, 7, 3), (16384, 64, 8), (16385, 64, 8), (90001, 256, 3)]


@pytest.mark.parametrize("masked", ["none", "some", "all"])
@pytest.mark.parametrize("T,E,K", SIZES)
def test_sort(T, E, K, masked):
    idx = _idx(1, T, E, K)
    mask = None
    if masked != "none":
        mask = torch.rand(T, generator=_gen(2), device="cuda") < (0.6 if masked == "some" else -1.0)
    offsets, slot = eat.expert_sort(idx, E, mask=mask)
    want = _sorted(idx, E, mask)
    assert torch.equal(offsets, want[0]) and torch.equal(slot, want[1])


@pytest.mark.parametrize("E", [1, 8, 256])
def test_sort_all_to_one_expert(E):
    """The fullest expert, in one block and in several."""
    for T, K in ((700, 4), (5000, 4), (40000, 4)):
        idx = torch.full((T, K), E - 1, dtype=torch.int32, device="cuda")
        offsets, slot = eat.expert_sort(idx, E)
        assert offsets.tolist() == [0] * E + [T * K]
        assert torch.equal(slot.flatten(), torch.arange(T * K, dtype=torch.int32, device="cuda"))


ROWS = [(1, 8, 2, 64, 0), (1, 64, 8, 2048, 0), (3, 3, 16, 7, 0), (70, 8, 2, 256, 1), (70, 60, 4, 1408, 0),
        (33, 5, 3, 1001, 0), (700, 64, 8, 320, 0), (2, 2, 1, 65536, 0), (130, 16, 4, 2056, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,K,d,off", ROWS)
def test_gather(T, E, K, d, off, dtype):
    idx = _idx(3, T, E, K)
    offsets, slot, entry = _sorted(idx, E)
    x = _offset(_randn(4, T, d).to(dtype), off)
    x[0, 0] = NAN
    rows = eat.expert_gather(x, slot, offsets)
    want = torch.zeros(T * K, d, dtype=dtype, device="cuda")
    want[:len(entry)] = x[entry // K]
    assert torch.equal(rows.nan_to_num(7), want.nan_to_num(7))
    assert torch.equal(rows.isnan(), want.isnan())
    # in e4m3: as the rows quantised afterwards
    q, scale = eat.expert_gather_fp8(x, slot, offsets)
    q2, scale2 = eat.quant_rows(want)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scale, scale2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("T,E,K,d,off", ROWS)
def test_combine(T, E, K, d, off, weights, dtype):
    idx = _idx(5, T, E, K)
    offsets, slot, entry = _sorted(idx, E)
    n = len(entry)
    rows = _offset(_randn(6, T * K, d).to(dtype), off)
    rows[n:] = NAN
    w = torch.rand(T, K, generator=_gen(7), device="cuda")
    w[slot < 0] = NAN
    y = eat.expert_combine(rows, slot, w if weights else None)
    f = (w.flatten()[entry] if weights else torch.ones(n, device="cuda")).double()[:, None]
    terms = f * rows[:n].double()
    want = torch.zeros(T, d, dtype=F64, device="cuda").index_add_(0, entry // K, terms)
    mag = torch.zeros_like(want).index_add_(0, entry // K, terms.abs())
    assert y.dtype == dtype
    assert ((y.double() - want).abs() <= _u(dtype) * want.abs() + 2 * K * U32 * mag).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,K,d,off", ROWS)
def test_combine_grad(T, E, K, d, off, dtype):
    idx = _idx(8, T, E, K)
    offsets, slot, entry = _sorted(idx, E)
    n = len(entry)
    rows = _offset(_randn(9, T * K, d).to(dtype), off)
    rows[n:] = NAN
    dy = _offset(_randn(10, T, d).to(dtype), off)
    w = torch.rand(T, K, generator=_gen(11), device="cuda")
    w[slot < 0] = NAN
    drows, dw = eat.expert_combine_grad(dy, rows, slot, offsets, w)
    # automatic differentiation of the plain form in 64 bits
    r64, w64 = rows[:n].double().requires_grad_(), w.flatten()[entry].double().requires_grad_()
    y = torch.zeros(T, d, dtype=F64, device="cuda").index_add(0, entry // K, w64[:, None] * r64)
    y.backward(dy.double())
    assert ((drows[:n].double() - r64.grad).abs() <= (_u(dtype) + U32) * r64.grad.abs()).all()
    assert (drows[n:] == 0).all()
    mag = (dy.double()[entry // K] * rows[:n].double()).abs().sum(1)
    got = dw.flatten()
    # (lanes' partial sums of d / 256 terms or fewer, joined by trees)
    assert ((got[entry].double() - w64.grad).abs() <= (d / 32 + 24) * U32 * mag).all()
    assert (dw[slot < 0] == 0).all()
    again = eat.expert_combine_grad(dy, rows, slot, offsets, w)
    assert torch.equal(again[0], drows) and torch.equal(again[1], dw)


def test_combine_grad_against_differences():
    """combine is linear in its rows and in its weights, so a step of any size gives the derivative; fp32
    sums of K d terms are off by at most (K + d) 2^-24 of the magnitudes."""
    T, E, K, d = 37, 5, 3, 68
    offsets, slot, entry = _sorted(_idx(51, T, E, K), E)
    n = len(entry)
    rows, dy, w = _randn(52, T * K, d), _randn(53, T, d), torch.rand(T, K, generator=_gen(54), device="cuda")
    e, ew = _randn(55, T * K, d), _randn(56, T, K)
    drows, dw = eat.expert_combine_grad(dy, rows, slot, offsets, w)
    y = eat.expert_combine(rows, slot, w).double()
    for moved, grad, step in ((eat.expert_combine(rows + e, slot, w), drows[:n], e[:n]),
                              (eat.expert_combine(rows, slot, w + ew), dw[slot >= 0], ew[slot >= 0])):
        change = ((moved.double() - y) * dy.double()).sum()
        want = (grad.double() * step.double()).sum()
        mag = ((moved.double().abs() + y.abs()) * dy.double().abs()).sum()
        assert (change - want).abs() <= 4 * (K + d) * U32 * mag
    # and without weights it is gather's transpose
    x, din = _randn(57, T, d), _randn(58, T * K, d)
    a = (eat.expert_gather(x, slot, offsets).double()[:n] * din.double()[:n]).sum()
    b = (eat.expert_combine(din, slot).double() * x.double()).sum()
    assert (a - b).abs() <= (K + d) * U32 * (x.abs().max() * din.abs().sum()).double()


# ------------------------------------------------------------------------------ e4m3 in blocks
def _scales64(top):
    return torch.where(top > 1e-35, top / 448.0, 1.0)


def _blocked(v, dim):
    """v padded with zeros to whole blocks of 128 along dim, split there: [..., blocks, 128, ...]."""
    n = v.shape[dim]
    pad = -n % 128
    if pad:
        v = torch.cat([v, v.new_zeros(*v.shape[:dim], pad, *v.shape[dim + 1:])], dim)
    return v.unflatten(dim, (-1, 128))


def _check_bytes(q, v, scale):
    """q are the e4m3 values of v / scale, rounded (the quotient is rounded to fp32 first)."""
    t = v / scale
    step = torch.maximum(t.abs() * 2.0 ** -4, torch.full_like(t, 2.0 ** -10))
    assert ((q.double() - t).abs() <= step + 4 * U32 * t.abs()).all()


def _check_rows(x, q, scale):
    M, K = x.shape
    v = x.double()
    want = _scales64(_blocked(v, 1).abs().amax(2)).t()
    assert scale.shape == want.shape
    assert ((scale.double() - want).abs() <= 2 * U32 * want).all()
    _check_bytes(q, v, scale.double().t().repeat_interleave(128, 1)[:, :K])


MATRICES = [(1, 1, 0), (1, 16, 0), (7, 128, 0), (8, 130, 0), (33, 2048, 0), (129, 257, 0), (300, 1408, 0),
            (5, 65536, 0), (64, 256, 1), (64, 256, 4)]


def _values(seed, M, K, dtype):
    """Rows and columns of very different size, a block of zeros, tiny ones."""
    x = _randn(seed, M, K) * torch.exp(3.0 * _randn(seed + 1, M, 1)) * torch.exp(3.0 * _randn(seed + 2, K))
    if M > 4:
        x[1] = 0
        x[2] *= 1e-36
        x[3] *= 1e30 / x[3].abs().max()
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,K,off", MATRICES)
def test_quant_rows(M, K, off, dtype):
    x = _offset(_values(12, M, K, dtype), off)
    _check_rows(x, *eat.quant_rows(x))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quotients_are_rounded_once(dtype):
    """Values half way between two e4m3 values, which bf16 quotients often are, go where the fp32 quotient
    goes."""
    x = _offset(_randn(17, 512, 2048).to(dtype), 0)
    q, scale = eat.quant_rows(x)
    s = _blocked(x.double(), 1).abs().amax(2) / 448.0
    assert ((scale.t() - s).abs() <= 2 * U32 * s).all()
    want = (x.float() / scale.t().repeat_interleave(128, 1)).to(E4M3)
    assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))


def test_quant_rows_special():
    x = _randn(13, 4, 256)
    x[0, 5], x[1, 200], x[2, 7] = NAN, INF, -INF
    q, scale = eat.quant_rows(x)
    v = q.float() * scale.t().repeat_interleave(128, 1)
    assert v[0, 5].isnan() and v[0].isnan().sum() == 1
    assert v[1, 128:].isnan().all() and v[1, :128].isfinite().all()
    assert v[2, :128].isnan().all() and v[3].isfinite().all()


SPLITS = [[5], [0, 3, 0, 0, 130, 1], [128, 32, 33, 0, 257], [0, 0, 0], [31, 1, 127, 129, 0, 64] * 6,
          [0] * 255 + [300], [1] * 256, [300, 0, 17, 513, 1]]


def _offsets(split):
    return torch.tensor([0] + split, device="cuda").cumsum(0).to(torch.int32)


def _column_blocks(split):
    """(first row, rows, first padded row) of each block."""
    out, row, padded = [], 0, 0
    for n in split:
        for i in range(0, n, 128):
            out.append((row + i, min(128, n - i), padded + i))
        row, padded = row + n, padded + -(-n // 32) * 32
    return out, padded


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K,off", [(1, 0), (128, 0), (400, 0), (2055, 0), (256, 1)])
@pytest.mark.parametrize("split", range(len(SPLITS)))
def test_quant_columns(split, K, off, dtype):
    split = SPLITS[split]
    R = sum(split)
    M = R + 37
    x = _offset(_values(14, M, K, dtype), off)
    x[R:] = NAN  # behind the last expert's rows
    offsets = _offsets(split)
    q, scale, cq, cscale = eat.quant_rows_columns(x, offsets)
    cq2, cscale2 = eat.quant_columns(x, offsets)
    blocks, padded = _column_blocks(split)
    assert cq.shape[0] >= padded and cscale.shape[0] >= len(blocks)
    for b, (row, n, p) in enumerate(blocks):
        v = x[row:row + n].double()
        want = _scales64(v.abs().amax(0))
        assert ((cscale[b].double() - want).abs() <= 2 * U32 * want).all()
        _check_bytes(cq[p:p + n], v, cscale[b].double())
        assert (cq[p + n:p + -(-n // 32) * 32].float() == 0).all()
    assert torch.equal(cq[:padded].view(torch.uint8), cq2[:padded].view(torch.uint8))
    assert torch.equal(cscale[:len(blocks)], cscale2[:len(blocks)])
    # and the rows
    x[R:] = 0
    q2, scale2 = eat.quant_rows(x)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scale, scale2)


@pytest.mark.parametrize("M,K", [(1, 16), (31, 100), (129, 256), (1000, 72)])
def test_quant_columns_of_all_rows(M, K):
    x = _values(15, M, K, BF16)
    q, scale, cq, cscale = eat.quant_rows_columns(x)
    assert cq.shape == (-(-M // 32) * 32, K) and cscale.shape == (-(-M // 128), K)
    _check_rows(x, q, scale)
    for b in range(-(-M // 128)):
        v = x[128 * b:128 * b + 128].double()
        _check_bytes(cq[128 * b:128 * b + len(v)], v, cscale[b].double())
    assert (cq[M:].float() == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,N,K,off", [(0, 1, 1, 0), (0, 128, 128, 0), (0, 100, 300, 0), (3, 257, 144, 0),
                                       (2, 512, 256, 1), (256, 16, 16, 0)])
def test_quant_tiles(E, N, K, off, dtype):
    w = _values(16, max(1, E) * N, K, dtype)
    w = _offset(w.view(E, N, K) if E else w, off)
    q, scale = eat.quant_tiles(w)
    v = w.double()
    want = _scales64(_blocked(_blocked(v, w.dim() - 2), w.dim()).abs().amax((-3, -1)))
    assert scale.shape == want.shape
    assert ((scale.double() - want).abs() <= 2 * U32 * want).all()
    s = scale.double().repeat_interleave(128, -2).repeat_interleave(128, -1)[..., :N, :K]
    _check_bytes(q, v, s)


# -------------------------------------------------------------------------------- products
def _of_rows(q, scale):
    return q.double() * scale.double().t().repeat_interleave(128, 1)[:, :q.shape[1]]


def _of_tiles(q, scale):
    s = scale.double().repeat_interleave(128, -2).repeat_interleave(128, -1)
    return q.double() * s[..., :q.shape[-2], :q.shape[-1]]


def _check_product(got, want, mag, blocks, dtype):
    """A block's sum in the tensor cores, the blocks' in fp32, two products of scales."""
    tol = _u(dtype) * want.abs() + (10 + blocks / 2 + 2) * 2.0 ** -23 * mag
    assert got.dtype == dtype
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (bad.nonzero()[:4], (got.double() - want).abs().max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (1, 4096, 2048), (2, 48, 4096), (16, 128, 128), (17, 130, 144),
                                   (33, 2816, 256), (100, 77, 1408), (129, 256, 272), (257, 512, 400),
                                   (300, 1024, 128), (777, 528, 640)])
def test_product(M, N, K, transposed, dtype):
    if transposed:
        N = -(-N // 16) * 16
    inner = N if transposed else K
    x = (_randn(21, M, inner) * torch.exp(_randn(22, inner))).to(BF16)
    w = (_randn(23, N, K) * torch.exp(_randn(24, N, 1))).to(BF16)
    (xq, xs), (wq, ws) = eat.quant_rows(x), eat.quant_tiles(w)
    y = eat.block_mm(xq, xs, wq, ws, transposed=transposed, dtype=dtype)
    a, b = _of_rows(xq, xs), _of_tiles(wq, ws)
    b = b if transposed else b.t()
    _check_product(y, a @ b, a.abs() @ b.abs(), -(-inner // 128), dtype)
    assert torch.equal(y, eat.block_mm(xq, xs, wq, ws, transposed=transposed, dtype=dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("split", range(len(SPLITS)))
@pytest.mark.parametrize("N,K", [(256, 128), (80, 272), (512, 400)])
def test_product_of_experts(split, N, K, transposed, dtype):
    split = SPLITS[split]
    E, R = len(split), sum(split)
    M, inner = R + 19, N if transposed else K
    x = (_randn(25, M, inner) * torch.exp(_randn(26, M, 1))).to(BF16)
    x[R:] = NAN
    w = (_randn(27, E, N, K) * torch.exp(_randn(28, E, N, 1))).to(BF16)
    if E > 2:
        w[1] = NAN  # reaches its own rows alone
    offsets = _offsets(split)
    (xq, xs), (wq, ws) = eat.quant_rows(x), eat.quant_tiles(w)
    y = eat.block_mm(xq, xs, wq, ws, offsets=offsets, transposed=transposed, dtype=dtype)
    a, b = _of_rows(xq, xs), _of_tiles(wq, ws)
    for e in range(E):
        lo, hi = offsets[e].item(), offsets[e + 1].item()
        if lo == hi:
            continue
        if E > 2 and e == 1:
            assert y[lo:hi].isnan().all()
            continue
        m = b[e] if transposed else b[e].t()
        _check_product(y[lo:hi], a[lo:hi] @ m, a[lo:hi].abs() @ m.abs(), -(-inner // 128), dtype)
    assert (y[R:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("split,cols,inner", [
    ([1500], 3008, 400), ([1500], 3008, 1680), ([2001], 2816, 272), ([90], 8192, 272), ([200], 8192, 144),
    ([300, 0, 517, 513, 1], 2816, 272), ([0, 900, 17, 2, 400], 2832, 1616), ([100, 90, 130] * 4, 2048, 272),
    ([40, 0, 55, 33] * 10, 2048, 144), ([700, 3] * 3, 2064, 1552)])
def test_products_of_every_tile(split, cols, inner, transposed, dtype):
    """Enough tiles of each kind: few and many rows an expert, short and long sums."""
    E, R = len(split), sum(split)
    M, N, K = R + 7, *((inner, cols) if transposed else (cols, inner))
    x, w = _randn(141, M, inner).to(BF16), _randn(142, E, N, K).to(BF16)
    x[R:] = NAN
    offsets = _offsets(split)
    (xq, xs), (wq, ws) = eat.quant_rows(x), eat.quant_tiles(w)
    y = eat.block_mm(xq, xs, wq, ws, offsets=offsets, transposed=transposed, dtype=dtype)
    a, b = _of_rows(xq, xs), _of_tiles(wq, ws)
    for e in range(E):
        r = slice(offsets[e].item(), offsets[e + 1].item())
        m = b[e] if transposed else b[e].t()
        _check_product(y[r], a[r] @ m, a[r].abs() @ m.abs(), -(-inner // 128), dtype)
    assert (y[R:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("split", range(len(SPLITS)))
@pytest.mark.parametrize("N,K", [(16, 16), (256, 128), (80, 272), (512, 400)])
def test_product_grad(split, N, K, dtype):
    split = SPLITS[split]
    E, R = len(split), sum(split)
    M = R + 3
    g, x = _randn(31, M, N).mul(1e-3).to(BF16), (_randn(32, M, K) * torch.exp(_randn(33, K))).to(BF16)
    g[R:], x[R:] = NAN, INF
    offsets = _offsets(split)
    (gq, gs), (xq, xs) = eat.quant_columns(g, offsets), eat.quant_columns(x, offsets)
    dw = eat.block_mm_grad(gq, gs, xq, xs, offsets=offsets, dtype=dtype)
    assert dw.shape == (E, N, K)
    blocks, _ = _column_blocks(split)
    b = 0
    for e, n in enumerate(split):
        want = torch.zeros(N, K, dtype=F64, device="cuda")
        mag = torch.zeros_like(want)
        for _ in range(0, n, 128):
            _, rows, p = blocks[b]
            u = gq[p:p + rows].double() * gs[b].double()
            v = xq[p:p + rows].double() * xs[b].double()
            want += u.t() @ v
            mag += u.abs().t() @ v.abs()
            b += 1
        _check_product(dw[e], want, mag, -(-n // 128), dtype)
    assert torch.equal(dw, eat.block_mm_grad(gq, gs, xq, xs, offsets=offsets, dtype=dtype))


@pytest.mark.parametrize("M,N,K", [(1, 16, 32), (100, 128, 144), (300, 272, 1040), (2000, 64, 256)])
def test_product_grad_of_all_rows(M, N, K):
    g, x = _randn(34, M, N).to(BF16), _randn(35, M, K).to(BF16)
    (gq, gs), (xq, xs) = eat.quant_columns(g), eat.quant_columns(x)
    dw = eat.block_mm_grad(gq, gs, xq, xs)
    u = gq.double() * gs.double().repeat_interleave(128, 0)[:len(gq)]
    v = xq.double() * xs.double().repeat_interleave(128, 0)[:len(xq)]
    _check_product(dw, u.t() @ v, u.abs().t() @ v.abs(), -(-M // 128), BF16)


def test_offsets_out_of_order_stay_in_the_buffers():
    """Offsets that no sort makes: the calls end, and leave what lies behind their outputs alone."""
    M, N, K = 96, 64, 128
    x, w = _randn(36, M, K).to(BF16), _randn(37, 4, N, K).to(BF16)
    (xq, xs), (wq, ws) = eat.quant_rows(x), eat.quant_tiles(w)
    for bad in ([0, 90, 10, 200, 96], [-5, 96, 0, 96, 0], [1 << 30, -7, 50, 3, 1 << 30], [96] * 5):
        o = torch.tensor(bad, dtype=torch.int32, device="cuda")
        y = torch.full((M + 8, N), 7.0, dtype=BF16, device="cuda")
        eat.eat_block_mm(xq, xs, wq, ws, o, 4, M, N, K, 0, y, eat.EAT_BF16)
        assert (y[M:] == 7).all()
        rows, blocks = eat.eat_quant_columns_rows(M, 4), eat.eat_quant_columns_blocks(M, 4)
        cq = torch.full((rows + 8, K), 7.0, device="cuda").to(E4M3)
        cs = torch.full((blocks + 1, K), 7.0, device="cuda")
        eat.eat_quant_columns(x, M, K, eat.EAT_BF16, o, 4, None, None, cq, cs)
        assert (cq[rows:].float() == 7).all() and (cs[blocks:] == 7).all()
        dw = torch.full((5, K, K), 7.0, device="cuda")
        eat.eat_block_mm_grad(cq, cs, cq, cs, o, 4, rows, blocks, K, K, dw, eat.EAT_F32)
        assert (dw[4] == 7).all()


# -------------------------------------------------------------------------- gated activation
GLU = [(1, 1, 0), (1, 16, 0), (3, 129, 0), (8, 14336, 0), (33, 1408, 0), (700, 256, 0), (5, 100, 1), (2, 65536, 0)]


def _glu64(gu):
    gate, up = gu.double().chunk(2, 1)
    return gate, up, gate * torch.sigmoid(gate) * up


def _glu_tol(gate, up, h):
    # the sigmoid within 3 2^-23 + |gate| 2^-24 of itself, and two products
    return (8 + gate.abs()) * U32 * h.abs()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,F,off", GLU)
def test_swiglu(R, F, off, dtype):
    gu = _offset((4.0 * _randn(41, R, 2 * F)).to(dtype), off)
    if R > 2:
        gu[1, :F], gu[2, :F] = 60.0, -60.0
    h = eat.swiglu(gu)
    gate, up, want = _glu64(gu)
    assert ((h.double() - want).abs() <= _u(dtype) * want.abs() + _glu_tol(gate, up, want) + 1e-38).all()
    q, scale = eat.swiglu_fp8(gu)
    ref = _scales64(_blocked(want, 1).abs().amax(2)).t()
    assert ((scale.double() - ref).abs() <= (80 * U32) * ref).all()
    s = scale.double().t().repeat_interleave(128, 1)[:, :F]
    t = want / s
    step = torch.maximum(t.abs() * 2.0 ** -4, torch.full_like(t, 2.0 ** -10))
    assert ((q.double() - t).abs() <= step + _glu_tol(gate, up, want) / s + 4 * U32 * t.abs()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_swiglu_special(dtype):
    """Far negative and positive gates, infinities and NaN."""
    gate = torch.tensor([-1e4, -200.0, -88.0, 0.0, 88.0, 1e4, INF, -INF, NAN], device="cuda")
    gu = torch.cat([gate, torch.ones_like(gate)])[None].to(dtype)
    h = eat.swiglu(gu)[0].float()
    assert h[:2].tolist() == [0.0, 0.0] and abs(h[2]) < 1e-35 and h[3] == 0
    assert h[4] == gu[0, 4] and h[5] == gu[0, 5] and h[6] == INF and h[8].isnan()
    d = eat.swiglu_grad(gu, torch.ones(1, 9, dtype=dtype, device="cuda"))[0].float()
    assert (d[:6].isfinite()).all() and (d[9:15].isfinite()).all()
    assert d[0] == 0 and d[1] == 0 and d[3] == 0.5 and d[5] == 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,F,off", GLU)
def test_swiglu_grad(R, F, off, dtype):
    gu = _offset((4.0 * _randn(42, R, 2 * F)).to(dtype), off)
    dh = _offset(_randn(43, R, F).to(dtype), off)
    dgu = eat.swiglu_grad(gu, dh)
    v = gu.double().requires_grad_()
    _glu64(v)[2].backward(dh.double())
    gate, up, _ = _glu64(gu)
    s = torch.sigmoid(gate)
    # magnitudes of what is added in 1 + gate (1 - s)
    mag = torch.cat([dh.double().abs() * up.abs() * s * (1 + gate.abs() * (1 - s) + gate.abs() * s),
                     (dh.double() * gate * s).abs()], 1)
    tol = _u(dtype) * v.grad.abs() + (12 + gate.abs().repeat(1, 2)) * U32 * mag
    assert ((dgu.double() - v.grad).abs() <= tol + 1e-38).all()


def test_swiglu_grad_in_place():
    gu, dh = _randn(46, 33, 400).to(BF16), _randn(47, 33, 200).to(BF16)
    want = eat.swiglu_grad(gu, dh)
    eat.eat_swiglu_grad(gu, dh, 33, 200, eat.EAT_BF16, gu)
    assert torch.equal(gu, want)


def test_swiglu_grad_against_differences():
    gu, dh = 2.0 * _randn(44, 6, 64), _randn(45, 6, 32)
    dgu = eat.swiglu_grad(gu, dh)
    step = 2.0 ** -6
    for i in (0, 7, 31, 32, 63):
        e = torch.zeros(64, device="cuda")
        e[i] = step
        dif = ((eat.swiglu(gu + e).double() - eat.swiglu(gu - e).double()) * dh.double()).sum(1) / (2 * step)
        # the third derivative is at most |up| in magnitude; h is at most |gate up|, off by 2^-21 of it
        top = gu.abs().amax(1)
        tol = dh.abs().sum(1) * (top * step ** 2 / 6 + (top + step) ** 2 * 2.0 ** -21 / step)
        assert ((dgu[:, i].double() - dif).abs() <= tol).all()


# ------------------------------------------------------------------------------- as they are used
def _layer(idx, w, x, w1, w2, mask, dy):
    """Experts of a router's choice, forward and backward; every tensor of the run."""
    E = w1.shape[0]
    o, slot = eat.expert_sort(idx, E, mask=mask)
    rows = eat.expert_gather(x, slot, o)
    xq, xs, xcq, xcs = eat.quant_rows_columns(rows, o)
    w1q, w1s = eat.quant_tiles(w1)
    gu = eat.block_mm(xq, xs, w1q, w1s, offsets=o)
    hq, hs = eat.swiglu_fp8(gu)
    w2q, w2s = eat.quant_tiles(w2)
    out = eat.block_mm(hq, hs, w2q, w2s, offsets=o)
    y = eat.expert_combine(out, slot, w)
    dout, dw = eat.expert_combine_grad(dy, out, slot, o, w)
    gq, gs, gcq, gcs = eat.quant_rows_columns(dout, o)
    hcq, hcs = eat.quant_columns(eat.swiglu(gu), o)
    dh = eat.block_mm(gq, gs, w2q, w2s, offsets=o, transposed=True)
    dw2 = eat.block_mm_grad(gcq, gcs, hcq, hcs, offsets=o)
    dgu = eat.swiglu_grad(gu, dh)
    dq, ds, dcq, dcs = eat.quant_rows_columns(dgu, o)
    drows = eat.block_mm(dq, ds, w1q, w1s, offsets=o, transposed=True)
    dw1 = eat.block_mm_grad(dcq, dcs, xcq, xcs, offsets=o)
    dx = eat.expert_combine(drows, slot)
    return dict(y=y, dx=dx, dw=dw, dw1=dw1, dw2=dw2)


def _layer64(idx, w, x, w1, w2, mask, dy):
    """The same without any e4m3, by automatic differentiation in 64 bits."""
    E, F, K = w1.shape[0], w2.shape[2], idx.shape[1]
    x, w, w1, w2 = (t.double().requires_grad_() for t in (x, w, w1, w2))
    y = torch.zeros_like(x)
    for e in range(E):
        live = idx == e
        if mask is not None:
            live &= mask[:, None]
        t, k = live.nonzero(as_tuple=True)
        gu = x[t] @ w1[e].t()
        h = torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]
        y = y.index_add(0, t, w[t, k][:, None] * (h @ w2[e].t()))
    y.backward(dy.double())
    return dict(y=y.detach(), dx=x.grad, dw=w.grad, dw1=w1.grad, dw2=w2.grad)


def _layer_inputs(seed, T, E, K, d, F):
    idx = _idx(seed, T, E, K)
    idx[0, 0] = 0
    w = torch.rand(T, K, generator=_gen(seed + 1), device="cuda")
    x, dy = _randn(seed + 2, T, d).to(BF16), _randn(seed + 3, T, d).to(BF16)
    w1 = (_randn(seed + 4, E, 2 * F, d) / d ** 0.5).to(BF16)
    w2 = (_randn(seed + 5, E, d, F) / F ** 0.5).to(BF16)
    mask = torch.rand(T, generator=_gen(seed + 6), device="cuda") < 0.8
    mask[0] = True
    return idx, w, x, w1, w2, mask, dy


@pytest.mark.parametrize("T,E,K,d,F", [(1, 8, 2, 256, 512), (130, 8, 2, 256, 144), (600, 12, 4, 400, 272)])
def test_layer(T, E, K, d, F):
    """A run of them: each result is as far from the unquantised one as roundings to e4m3 (2^-4 at
    most, independent of each other, at most five on the way to any output) make it."""
    a = _layer_inputs(60, T, E, K, d, F)
    got, want = _layer(*a), _layer64(*a)
    for n, v in want.items():
        err = ((got[n].double() - v).norm() / v.norm()).item()
        assert err <= 5 ** 0.5 * 2.0 ** -4, (n, err)


def test_layer_captured_and_replayed():
    a, b = (_layer_inputs(s, 200, 8, 2, 256, 144) for s in (70, 80))
    buf = [t.clone() for t in a]
    eager = [_layer(*t) for t in (a, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(*buf)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(*buf)
    for want, src in ((eager[0], a), (eager[1], b), (eager[0], a)):
        for t, s in zip(buf, src):
            t.copy_(s)
        graph.replay()
        for n in want:
            assert torch.equal(out[n], want[n]), n


def test_layer_on_two_streams():
    args = [_layer_inputs(s, 300, 8, 2, 256, 144) for s in (90, 100)]
    want = [_layer(*a) for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_layer(*args[i]))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for r in g:
            for n in w:
                assert torch.equal(r[n], w[n]), n


@pytest.mark.parametrize("split", [[128], [128, 0, 256], [512, 128], [0, 128] * 40])
def test_products_of_integers_are_exact(split):
    """Powers of two up to 4, and 448 once in every row, column and tile of a block: the scales are 1, every
    product and sum is a whole number below 2^24, and all three products come out exactly."""
    E, M, N, K = len(split), sum(split), 256, 384

    def whole(seed, *shape):
        v = 2.0 ** torch.randint(0, 3, shape, generator=_gen(seed), device="cuda")
        v *= torch.randint(-1, 2, shape, generator=_gen(seed + 1), device="cuda")
        i, j = (torch.arange(n, device="cuda") % 128 for n in shape[-2:])
        return torch.where(i[:, None] == j, 448.0, v).to(BF16)

    x, g, w = whole(131, M, K), whole(133, M, N), whole(135, E, N, K)
    o = _offsets(split)
    (wq, ws), (xq, xs, xcq, xcs) = eat.quant_tiles(w), eat.quant_rows_columns(x, o)
    gq, gs, gcq, gcs = eat.quant_rows_columns(g, o)
    blocks = M // 128
    assert (ws == 1).all() and (xs == 1).all() and (xcs[:blocks] == 1).all() and (gcs[:blocks] == 1).all()
    y = eat.block_mm(xq, xs, wq, ws, offsets=o, dtype=F32)
    dx = eat.block_mm(gq, gs, wq, ws, offsets=o, transposed=True, dtype=F32)
    dw = eat.block_mm_grad(gcq, gcs, xcq, xcs, offsets=o, dtype=F32)
    for e in range(E):
        r = slice(o[e].item(), o[e + 1].item())
        assert torch.equal(y[r].double(), x[r].double() @ w[e].double().t())
        assert torch.equal(dx[r].double(), g[r].double() @ w[e].double())
        assert torch.equal(dw[e].double(), g[r].double().t() @ x[r].double())


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("N,K", [(65536, 128), (128, 65536)])
def test_widest_products(N, K, transposed):
    M, inner = 130, N if transposed else K
    x, w = _randn(111, M, inner).to(BF16), _randn(112, N, K).to(BF16)
    (xq, xs), (wq, ws) = eat.quant_rows(x), eat.quant_tiles(w)
    a, b = _of_rows(xq, xs), _of_tiles(wq, ws)
    b = b if transposed else b.t()
    for rows in (M, 5):
        y = eat.block_mm(xq[:rows], xs[:, :rows].contiguous(), wq, ws, transposed=transposed, dtype=F32)
        _check_product(y, a[:rows] @ b, a[:rows].abs() @ b.abs(), -(-inner // 128), F32)


def test_rows_far_into_a_buffer():
    """Elements and bytes whose offsets pass 32 bits: the last rows as in a call of their own."""
    T, d, n = 70000, 65536, 112  # (the last 112 rows are a block of columns)
    x = torch.empty(T, d, dtype=BF16, device="cuda").normal_(generator=_gen(121))
    idx = (torch.arange(T, device="cuda") % 2).to(torch.int32)[:, None].contiguous()
    offsets, slot = eat.expert_sort(idx, 2)
    rows = eat.expert_gather(x, slot, offsets)
    assert torch.equal(rows[-3:], x[-5::2]) and torch.equal(rows[T // 2 - 2:T // 2], x[-4::2])
    assert torch.equal(eat.expert_combine(rows, slot), x)
    drows, dw = eat.expert_combine_grad(x, rows, slot, offsets, torch.ones(T, 1, device="cuda"))
    assert torch.equal(drows[-3:], rows[-3:])
    assert ((dw[-2:, 0] - x[-2:].double().square().sum(1)).abs() < 1e-3 * d).all()
    del rows, drows
    q, scale = eat.quant_rows(x)
    q1, scale1 = eat.quant_rows(x[-n:])
    assert torch.equal(q[-n:].view(torch.uint8), q1.view(torch.uint8))
    assert torch.equal(scale[:, -n:], scale1)
    w, wt = (eat.quant_tiles(_randn(s, 16, d).to(BF16)) for s in (122, 123))
    y = eat.block_mm(q, scale, *w)
    a, b = _of_rows(q[-130:], scale[:, -130:]), _of_tiles(*w).t()
    _check_product(y[-130:], a @ b, a.abs() @ b.abs(), d // 128, BF16)
    _, _, cq, cscale = eat.quant_rows_columns(x)
    c1, cs1 = eat.quant_columns(x[-n:])
    assert torch.equal(cq[T - n:].view(torch.uint8), c1.view(torch.uint8))  # (both padded to 128 rows)
    assert torch.equal(cscale[-1], cs1[0])
    gq, gs = eat.quant_columns(y)
    dw = eat.block_mm_grad(gq, gs, cq, cscale)
    assert dw.shape == (16, d) and dw.isfinite().all()
    del cq, cscale
    yq, ys = eat.quant_rows(y)
    back = eat.block_mm(yq, ys, *wt, transposed=True)
    a, b = _of_rows(yq[-130:], ys[:, -130:]), _of_tiles(*wt)
    _check_product(back[-130:], a @ b, a.abs() @ b.abs(), 1, BF16)
    del back, q
    gu = x.view(T // 2, 2 * d)
    h = eat.swiglu(gu)
    assert torch.equal(h[-3:], eat.swiglu(gu[-3:]))
    dgu = eat.swiglu_grad(gu, h)
    assert torch.equal(dgu[-3:], eat.swiglu_grad(gu[-3:], h[-3:]))
    h8, s8 = eat.swiglu_fp8(gu)
    h1, s1 = eat.swiglu_fp8(gu[-3:])
    assert torch.equal(h8[-3:].view(torch.uint8), h1.view(torch.uint8)) and torch.equal(s8[:, -3:], s1)


def test_routing_of_a_layer_feeds_the_sort():
    """idx and w as EatLayer.route writes them."""
    from paper_2609_33614_gb300 import workloads as W
    lw = W.make_layer(W.TOY)
    layer = eat.EatLayer.from_workload(lw, max_tokens=96)
    idx, w, k = layer.route(W.make_tokens(W.TOY, 96, step=0).cuda())
    offsets, slot = eat.expert_sort(idx, lw.shape.n_experts)
    want = _sorted(idx, lw.shape.n_experts)
    assert torch.equal(offsets, want[0]) and torch.equal(slot, want[1])
    assert offsets[-1] == k.sum()
    rows = eat.expert_gather(W.make_tokens(W.TOY, 96, step=0).cuda(), slot, offsets)
    y = eat.expert_combine(rows, slot, w)
    x = W.make_tokens(W.TOY, 96, step=0).cuda()
    torch.testing.assert_close(y, x * w.sum(1, keepdim=True), rtol=1e-5, atol=1e-6)
    layer.close()
