"""GPU: RMS norm, balance loss and vocabulary cross entropy, with their gradients, against plain
64-bit implementations.

Tolerances.  bf16 has 8 significant bits (steps of 2^-7 in [1, 2)), so one rounding moves a value by
at most u16 = 2^-8 of itself; fp32 sums and functions stay within a few 2^-23 of the sum of magnitudes.  Tensor-core sums
truncate: a logit moves by at most (d / 16 + 2) 2^-23 sum |x w|.
"""
import math

import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -23
EPS = 1e-6


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
    buf = torch.zeros(t.numel() + 64, dtype=t.dtype, device="cuda")
    v = buf[n:n + t.numel()].view(t.shape)
    v.copy_(t)
    return v


# ------------------------------------------------------------------------------------ RMS norm
NORM_SIZES = [(1, 1), (1, 7), (2, 64), (5, 255), (33, 256), (64, 1408), (700, 2048), (3, 4096),
              (9, 8192), (2, 8200), (1, 65536), (4099, 72)]


def _norm64(x, r, gamma):
    s = x.double() + (0.0 if r is None else r.double())
    return s, s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * gamma.double()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("T,d", NORM_SIZES)
def test_rms_norm(T, d, off, residual, dtype):
    x = _offset((3.0 * _randn(1, T, d)).to(dtype), off)
    r = _offset(_randn(2, T, d).to(dtype), off) if residual else None
    gamma = _offset(1.0 + 0.2 * _randn(3, d), off)
    if T > 2:
        x[1] = 0
        if residual:
            r[1] = 0
    y, h = eat.rms_norm(x, gamma, EPS, residual=r)
    s, want = _norm64(x, r, gamma)
    u = U16 if dtype == torch.bfloat16 else 0.0
    # one rounding of the sum when stored; fp32 sum, mean, root, two products
    assert ((h.double() - s).abs() <= (u + U32) * s.abs()).all()
    assert ((y.double() - want).abs() <= (u + 16 * U32) * want.abs() + 1e-30).all()
    # the e4m3 form: 4 significant bits above 2^-6, steps of 2^-9 below, of the row's scale
    q, scale, h8 = eat.rms_norm_fp8(x, gamma, EPS, residual=r)
    top = want.abs().amax(1)
    ref = torch.where(top > 0, top / 448.0, 1.0)
    assert ((scale.double() - ref).abs() <= 16 * U32 * ref).all()
    assert torch.equal(h8, h)
    v = want / ref[:, None]
    step = torch.maximum(v.abs() * 2.0 ** -4, torch.full_like(v, 2.0 ** -10))
    assert ((q.double() - v).abs() <= step * (1 + 1e-5) + 1e-4 * step).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [100, 1024])
def test_rms_norm_in_place_and_special_rows(d, dtype):
    """h may be x or the residual; NaN and infinities stay in their row; tiny and huge rows."""
    T = 6
    x, r = _randn(4, T, d).to(dtype), _randn(5, T, d).to(dtype)
    x[1, 3] = math.nan
    x[2, 5] = math.inf
    x[3] *= 1e-18
    r[3] = 0
    x[4] *= 1e15
    gamma = 1.0 + 0.2 * _randn(6, d)
    y0, h0 = eat.rms_norm(x, gamma, EPS, residual=r)
    q0, s0, _ = eat.rms_norm_fp8(x, gamma, EPS, residual=r)
    code = eat.EAT_BF16 if dtype == torch.bfloat16 else eat.EAT_F32
    for into_x in (True, False):
        a, b = x.clone(), r.clone()
        y = torch.empty_like(a)
        h = a if into_x else b
        eat.eat_rms_norm(a, b, T, d, code, gamma, EPS, h, y, code)
        assert torch.equal(h.nan_to_num(7), h0.nan_to_num(7))
        assert torch.equal(y.nan_to_num(7), y0.nan_to_num(7))
    assert y0[1].isnan().all() and y0[[0, 3, 4, 5]].isfinite().all()
    v0 = q0.float() * s0[:, None]
    assert v0[1].isnan().all() and v0[[0, 3, 4, 5]].isfinite().all()
    _, want = _norm64(x, r, gamma)
    u = U16 if dtype == torch.bfloat16 else 0.0
    for t in (0, 3, 4, 5):
        assert ((y0[t].double() - want[t]).abs() <= (u + 16 * U32) * want[t].abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dres", [False, True])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("T,d", NORM_SIZES)
def test_rms_norm_grad(T, d, off, dres, dtype):
    h = _offset((2.0 * _randn(11, T, d)).to(dtype), off)
    dy = _offset(_randn(12, T, d).to(dtype), off)
    dr = _offset(_randn(13, T, d).to(dtype), off) if dres else None
    gamma = _offset(1.0 + 0.2 * _randn(14, d), off)
    dx, dgamma = eat.rms_norm_grad(h, gamma, EPS, dy, dres=dr)
    # the formula by automatic differentiation in 64 bits
    s = h.double().requires_grad_()
    g = gamma.double().requires_grad_()
    (s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * g).backward(dy.double())
    want = s.grad + (0.0 if dr is None else dr.double())
    # magnitudes of the terms that are added
    rstd = 1.0 / (h.double().square().mean(1, keepdim=True) + EPS).sqrt()
    n, gd = h.double() * rstd, (gamma * dy).double()
    mag = rstd * (gd.abs() + n.abs() * (gd * n).abs().mean(1, keepdim=True))
    mag = mag + (0.0 if dr is None else dr.double().abs())
    u = U16 if dtype == torch.bfloat16 else 0.0
    assert ((dx.double() - want).abs() <= u * want.abs() + 32 * U32 * mag + 1e-30).all()
    # a sum of T terms in fp32: partial sums of at most a few hundred terms, joined
    gm = (dy.double() * n).abs().sum(0)
    assert ((dgamma.double() - g.grad).abs() <= (16 + T ** 0.5) * U32 * gm + 1e-30).all()
    again = eat.rms_norm_grad(h, gamma, EPS, dy, dres=dr)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma)


def test_rms_norm_grad_against_differences():
    T, d = 5, 96
    x, gamma, dy = _randn(21, T, d), 1.0 + 0.2 * _randn(22, d), _randn(23, T, d)
    ux, ug = _randn(24, T, d), _randn(25, d)
    dx, dgamma = eat.rms_norm_grad(x, gamma, EPS, dy)
    f = lambda a, b: (eat.rms_norm(a, b, EPS)[0].double() * dy.double()).sum()
    e = 2.0 ** -7
    # the third-order term of a central difference is about e^2 = 6e-5 of the terms' size
    size = (dx.double() * ux.double()).abs().sum()
    num = (f(x + e * ux, gamma) - f(x - e * ux, gamma)) / (2 * e)
    assert abs(num - (dx.double() * ux.double()).sum()) <= 1e-3 * size
    size = (dgamma.double() * ug.double()).abs().sum()
    num = (f(x, gamma + e * ug) - f(x, gamma - e * ug)) / (2 * e)
    assert abs(num - (dgamma.double() * ug.double()).sum()) <= 1e-3 * size


@pytest.mark.parametrize("alias", ["dy", "dres"])
@pytest.mark.parametrize("d", [90, 512])
def test_rms_norm_grad_in_place(d, alias):
    T = 700
    h, dy, dres = (_randn(31 + i, T, d).to(torch.bfloat16) for i in range(3))
    gamma = 1.0 + 0.2 * _randn(34, d)
    want = eat.rms_norm_grad(h, gamma, EPS, dy, dres=dres)
    dgamma = torch.empty(d, device="cuda")
    work = torch.empty(eat.eat_rms_norm_grad_workspace(T, d), dtype=torch.uint8, device="cuda")
    dx = dy if alias == "dy" else dres
    eat.eat_rms_norm_grad(h, T, d, eat.EAT_BF16, gamma, EPS, dy, dres, dx, dgamma, work)
    assert torch.equal(dx, want[0]) and torch.equal(dgamma, want[1])


# -------------------------------------------------------------------------------- balance loss
def _balance64(logits, idx, mask, g):
    T, E = logits.shape
    on = torch.ones(T, dtype=torch.bool, device="cuda") if mask is None else mask.bool()
    live = idx[on].flatten()
    live = live[(live >= 0) & (live < E)]
    counts = torch.bincount(live.long(), minlength=E)
    z = logits[on].double().requires_grad_()
    d = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    if on.sum() == 0 or counts.sum() == 0:
        return torch.zeros((), dtype=torch.float64), counts, on.sum(), d
    loss = E * (torch.softmax(z, 1).mean(0) * (counts.double() / counts.sum())).sum()
    (g * loss).backward()
    d[on] = z.grad
    return loss.detach(), counts, on.sum(), d


def _selected(T, E, K, seed):
    idx = torch.randn(T, E, generator=_gen(seed), device="cuda").topk(K, 1).indices.sort(1).values
    n = torch.randint(0, K + 1, (T, 1), generator=_gen(seed + 1), device="cuda")
    return torch.where(torch.arange(K, device="cuda") < n, idx, -1).to(torch.int32).contiguous()


def _check_balance(logits, idx, mask, g=0.37):
    T, E = logits.shape
    loss, counts, n = eat.balance_loss(logits, idx, mask=mask)
    gt = torch.full((1,), g, device="cuda")
    d = eat.balance_grad(logits, counts, n, gt, mask=mask)
    want, c64, n64, d64 = _balance64(logits, idx, mask, gt.double()[0])
    assert torch.equal(counts.long(), c64) and int(n) == int(n64)
    # p within 16 units of fp32 (exponential of a difference of at most ~20), sums of positive terms
    assert abs(float(loss) - float(want)) <= 64 * U32 * abs(float(want))
    p = torch.softmax(logits.double(), 1).nan_to_num(0.0)
    f = c64.double() / max(1, int(c64.sum()))
    mag = g * E / max(1, int(n)) * p * (f + (p * f).sum(1, keepdim=True))
    assert ((d.double() - d64).abs() <= 64 * U32 * mag + 1e-30).all()
    assert torch.equal(eat.balance_loss(logits, idx, mask=mask)[0], loss)
    return d


@pytest.mark.parametrize("masked", [None, 0.0, 0.5, 1.0])
@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (1, 8, 2), (2, 3, 1), (31, 8, 2), (33, 33, 4),
                                   (257, 60, 4), (1000, 64, 8), (513, 255, 16), (40, 256, 6),
                                   (20011, 64, 6)])
def test_balance(T, E, K, masked):
    logits = 2.0 * _randn(41, T, E)
    mask = None if masked is None else \
        torch.rand(T, generator=_gen(42), device="cuda") >= masked
    _check_balance(logits, _selected(T, E, K, 43), mask)


def test_balance_masked_rows_hold_anything():
    """NaN, infinities and lowest values in rows that do not count; entries outside [0, E)."""
    T, E, K = 130, 24, 3
    logits, idx = _randn(44, T, E), _selected(T, E, K, 45)
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[::3] = False
    logits[::3] = math.nan
    logits[3] = math.inf
    logits[6] = torch.finfo(torch.float32).min
    idx[::3] = 5
    idx[1, 0], idx[2, 0] = E, -(1 << 31)
    logits[4, 2:] = torch.finfo(torch.float32).min  # counted: all but two experts ruled out
    logits[5, 1:] = -math.inf
    d = _check_balance(logits, idx, mask)
    assert (d[::3] == 0).all() and d.isfinite().all()


def test_balance_no_selection():
    T, E = 50, 16
    idx = torch.full((T, 2), -1, dtype=torch.int32, device="cuda")
    d = _check_balance(_randn(46, T, E), idx, None)
    assert (d == 0).all()


def test_balance_grad_against_differences():
    T, E, K = 40, 12, 2
    logits, idx, u = _randn(47, T, E), _selected(T, E, K, 48), _randn(49, T, E)
    _, counts, n = eat.balance_loss(logits, idx)
    d = eat.balance_grad(logits, counts, n, torch.ones(1, device="cuda"))
    e = 2.0 ** -5
    num = (eat.balance_loss(logits + e * u, idx)[0] - eat.balance_loss(logits - e * u, idx)[0]) / (2 * e)
    # e^2 = 1e-3 of third-order terms, and 2 x 2^-23 of the loss (about 1) over 2 e
    size = (d.double() * u.double()).abs().sum()
    assert abs(float(num) - float((d * u).sum())) <= 2e-3 * float(size) + 4 * U32 / e


def test_balance_grad_in_place():
    T, E = 77, 40
    logits, idx = _randn(50, T, E), _selected(T, E, 2, 51)
    _, counts, n = eat.balance_loss(logits, idx)
    g = torch.ones(1, device="cuda")
    want = eat.balance_grad(logits, counts, n, g)
    eat.eat_balance_grad(logits, T, E, None, counts, n, g, logits)
    assert torch.equal(logits, want)


# ------------------------------------------------------------------------- vocabulary head
def _e4m3_rows(w):
    amax = w.abs().amax(1)
    s = torch.where(amax > 0, amax / 448.0, 1.0)
    return (w / s[:, None]).to(torch.float8_e4m3fn), s


def _head_case(T, V, d, seed, std=0.05, ignored=0.2):
    w = std * _randn(seed, V, d)
    y = torch.randint(0, V, (T,), generator=_gen(seed + 1), device="cuda")
    lean = 8.0 * torch.rand(T, 1, generator=_gen(seed + 2), device="cuda")
    x = _randn(seed + 3, T, d) + lean * w[y] / w[y].square().sum(1, keepdim=True)
    drop = torch.rand(T, generator=_gen(seed + 4), device="cuda") < ignored
    drop[0] = False
    return x, w, torch.where(drop, -1 - y, y).to(torch.int32)


def _check_nll(x64, w64, target, nll, lse):
    V, d = w64.shape
    on = (target >= 0) & (target < V)
    x, y = x64[on], target[on].long()[:, None]
    logits = x @ w64.T
    ref = torch.logsumexp(logits, 1)
    others = logits.scatter(1, y, -math.inf)
    r = torch.logsumexp(others, 1) - logits.gather(1, y)[:, 0]
    want = torch.nn.functional.softplus(r)
    # a logit's truncated sum, and the exponentials' and logarithms' roundings
    dl = (d / 16 + 2) * U32 * (x.abs() @ w64.abs().T).amax(1) + 8 * U32 * (1 + logits.abs().amax(1))
    # nll = log(1 + exp r): |d nll| <= (1 - exp(-nll)) |dr|, and 2 dl is a bound of |dr|
    assert ((nll[on].double() - want).abs() <= 2 * dl * (1 - torch.exp(-want)) + 4 * U32 * want
            + 1e-30).all()
    assert ((lse[on].double() - ref).abs() <= 2 * dl).all()
    neg, big = target < 0, target >= V
    assert (nll[neg] == 0).all() and (lse[neg] == 0).all()
    assert nll[big].isnan().all() and lse[big].isnan().all()


HEAD_SIZES = [(1, 1, 64), (1, 2, 64), (3, 127, 128), (2, 129, 320), (7, 5003, 256),
              (16, 1000, 1408), (17, 2049, 64), (33, 300, 512), (64, 40000, 256),
              (100, 777, 1024), (128, 4096, 192), (129, 257, 256), (255, 512, 448),
              (257, 1025, 64), (513, 3001, 576), (1000, 20011, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,V,d", HEAD_SIZES)
def test_head_nll(T, V, d, dtype):
    x, w, target = _head_case(T, V, d, 61)
    if T > 6:
        target[3] = V      # out of range
        target[4] = -(1 << 31)
    if dtype == "bf16":
        x, w, xs, ws = x.bfloat16(), w.bfloat16(), None, None
        x64, w64 = x.double(), w.double()
        if T > 6:
            x[4] = math.nan  # an ignored token holds anything
    else:
        (x, xs), (w, ws) = _e4m3_rows(x), _e4m3_rows(w)
        x64, w64 = x.double() * xs.double()[:, None], w.double() * ws.double()[:, None]
        if T > 6:
            xs[4] = math.nan
    head = eat.EatHead(w, T + 5, w_scale=ws)
    nll, lse = head.nll(x, target, x_scale=xs)
    _check_nll(x64, w64, target, nll, lse)
    # fewer tokens on the same handle, and without lse
    n = (T + 1) // 2
    out = torch.full((n + 1,), -7.0, device="cuda")
    eat.eat_head_nll(head.h, x, xs, n, target, out)
    _check_nll(x64[:n], w64, target[:n], out[:n], lse[:n])
    assert float(out[n]) == -7.0
    assert torch.equal(head.nll(x, target, x_scale=xs)[0].nan_to_num(9), nll.nan_to_num(9))
    head.close()


def test_head_nll_confident_and_hopeless_tokens():
    """nll from 1e-13 to hundreds, with its relative accuracy."""
    V, d, T = 700, 128, 40
    w = 0.2 * _randn(71, V, d)
    y = torch.randint(0, V, (T,), generator=_gen(72), device="cuda")
    gain = torch.linspace(-60, 40, T, device="cuda")[:, None]
    x = (0.1 * _randn(73, T, d) + gain * w[y] / w[y].square().sum(1, keepdim=True)).bfloat16()
    w = w.bfloat16()
    nll, lse = eat.EatHead(w, T).nll(x, y.to(torch.int32))
    assert float(nll.min()) < 1e-9 and float(nll.max()) > 30
    _check_nll(x.double(), w.double(), y.to(torch.int32), nll, lse)


@pytest.mark.parametrize("V", [900, 20000])
@pytest.mark.parametrize("T", [2, 20, 50, 100, 300])
def test_head_nll_rows_without_probability(T, V):
    """Vocabulary rows whose logit is -inf add nothing; as a target they cost infinitely much."""
    d, dead = 128, slice(100, 2 * V // 3)
    x, w, target = _head_case(T, V, d, 81, ignored=0.0)
    x[:, 0] = x[:, 0].abs() + 0.5
    x[1] = x[0]
    x, w = x.bfloat16(), w.bfloat16()
    live = torch.ones(V, dtype=torch.bool, device="cuda")
    live[dead] = False
    to_live = torch.cumsum(live, 0).to(torch.int32) - 1
    w[~live, 0] = -math.inf
    target = torch.where(live[target.long()], target, target % 100)
    target[1] = 300
    nll, lse = eat.EatHead(w, T).nll(x, target)
    on = torch.arange(T, device="cuda") != 1
    x64, w64 = x.double(), w[live].double()
    _check_nll(x64[on], w64, to_live[target[on].long()], nll[on], lse[on])
    assert float(nll[1]) == math.inf
    _check_nll(x64[:1], w64, to_live[target[:1].long()], nll[:1], lse[1:2])


def _grads64(x, w, target, g):
    V = w.shape[0]
    on = (target >= 0) & (target < V)
    p = torch.softmax(x[on] @ w.T, 1)
    rows = torch.arange(int(on.sum()), device="cuda")
    p[rows, target[on].long()] -= 1.0
    p *= g[on, None]
    dx = torch.zeros_like(x)
    dx[on] = p @ w
    ax = torch.zeros_like(x)
    ax[on] = p.abs() @ w.abs()
    return dx, p.T @ x[on], ax, p.abs().T @ x[on].abs()


def _check_grads(x, w, target, g, got, std_err):
    dx, dw, ax, aw = _grads64(x, w, target, g)
    # P as bf16 (u16), one more bf16 factor (u16), p's own error, the result's rounding (u16)
    for have, want, mag in ((got[0], dx, ax), (got[1], dw, aw)):
        bound = (2 * U16 + std_err) * mag * 1.01 + U16 * want.abs() + 1e-30
        assert ((have.double() - want).abs() <= bound).all()
    # the norm of the error: roundings do not add up
    for have, want in ((got[0], dx), (got[1], dw)):
        assert (have.double() - want).norm() <= U16 * want.norm() + 1e-30


GRAD_SIZES = [(1, 1, 64), (1, 130, 64), (5, 300, 128), (64, 1000, 256), (130, 257, 320),
              (257, 5003, 192), (300, 70000, 64), (1030, 2049, 576)]


@pytest.mark.parametrize("T,V,d", GRAD_SIZES)
def test_head_nll_grad(T, V, d):
    x, w, target = _head_case(T, V, d, 81)
    x, w = x.bfloat16(), w.bfloat16()
    g = torch.rand(T, generator=_gen(85), device="cuda") / T
    x64 = x.double()
    if T > 6:
        target[3], target[4] = V, -5
        x[3] = math.nan
        x[4] = math.inf
        g[4] = math.nan
        g[6] = 0.0
        x64[3:5] = 0
    head = eat.EatHead(w, T + 3, grad=True)
    nll, lse, dx, dw = head.nll_grad(x, target, g)
    assert torch.equal(nll.nan_to_num(9), head.nll_grad(x, target, g)[0].nan_to_num(9))
    _check_nll(x64, w.double(), target, nll, lse)
    dl = (d / 16 + 2) * U32 * float((x64.abs() @ w.double().abs().T).max())
    _check_grads(x64, w.double(), target, g.double(), (dx, dw), 4 * dl)
    off = (target < 0) | (target >= V)
    assert (dx[off] == 0).all() and dw.isfinite().all()
    again = head.nll_grad(x, target, g)
    assert torch.equal(again[2], dx) and torch.equal(again[3], dw)
    head.close()


def test_head_grad_no_token_counts():
    T, V, d = 70, 500, 128
    x, w, _ = _head_case(T, V, d, 91)
    target = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    x[:] = math.nan
    head = eat.EatHead(w.bfloat16(), T, grad=True)
    nll, lse, dx, dw = head.nll_grad(x.bfloat16(), target, torch.ones(T, device="cuda"))
    for t in (nll, lse, dx, dw):
        assert (t == 0).all()


def test_head_grad_far_tokens():
    """Tokens whose target is more than exp's range below the largest logit."""
    T, V, d = 140, 600, 64
    w = 0.5 * _randn(95, V, d)
    y = torch.randint(0, V, (T,), generator=_gen(96), device="cuda")
    x = 0.1 * _randn(97, T, d)
    x[::7] -= 200.0 * w[y[::7]] / w[y[::7]].square().sum(1, keepdim=True)
    x, w, target = x.bfloat16(), w.bfloat16(), y.to(torch.int32)
    g = torch.full((T,), 1.0 / T, device="cuda")
    head = eat.EatHead(w, T, grad=True)
    nll, lse, dx, dw = head.nll_grad(x, target, g)
    assert float(nll.max()) > 100
    _check_nll(x.double(), w.double(), target, nll, lse)
    dl = (d / 16 + 2) * U32 * float((x.double().abs() @ w.double().abs().T).max())
    _check_grads(x.double(), w.double(), target, g.double(), (dx, dw), 4 * dl)


@pytest.mark.parametrize("T,V", [(5, 300), (200, 300), (5, 512)])
def test_head_grad_all_logits_low(T, V):
    """Every logit of a token near -150: what the vocabulary's last tile pads counts as no row."""
    d = 128
    x, w, target = _head_case(T, V, d, 97)
    x, w = 0.1 * x, 0.02 * w
    x[::2, 0], w[:, 0] = -15.0, 10.0
    x, w = x.bfloat16(), w.bfloat16()
    g = _randn(98, T)
    nll, lse, dx, dw = eat.EatHead(w, T, grad=True).nll_grad(x, target, g)
    x64, w64 = x.double(), w.double()
    _check_nll(x64, w64, target, nll, lse)
    dl = (d / 16 + 4) * U32 * float((x64.abs() @ w64.abs().T).max())
    dx64, dw64, ax, aw = _grads64(x64, w64, target, g.double())
    for have, want, mag in ((dx, dx64, ax), (dw, dw64, aw)):  # (entry by entry: dx[:, 0] cancels)
        bound = (2 * U16 + 4 * dl) * mag * 1.01 + U16 * want.abs() + 1e-30
        assert ((have.double() - want).abs() <= bound).all()


def test_head_grad_against_differences():
    T, V, d = 60, 400, 128
    x, w, target = _head_case(T, V, d, 101, ignored=0.3)
    x, w = x.bfloat16(), w.bfloat16()
    g = torch.rand(T, generator=_gen(105), device="cuda")
    _, _, dx, dw = eat.EatHead(w, T, grad=True).nll_grad(x, target, g)

    def loss(a, b):
        return (eat.EatHead(b, T).nll(a, target)[0].double() * g.double()).sum()

    # steps to bf16 neighbours, so that both sides are exact inputs; logits move by about 0.05
    for what, u in (("x", _randn(106, T, d)), ("w", _randn(107, V, d))):
        if what == "x":
            hi, lo = (x + 0.1 * u).bfloat16(), (x - 0.1 * u).bfloat16()
            num, step, grad = loss(hi, w) - loss(lo, w), hi.double() - lo.double(), dx.double()
        else:
            hi, lo = (w + 0.005 * u).bfloat16(), (w - 0.005 * u).bfloat16()
            num, step, grad = loss(x, hi) - loss(x, lo), hi.double() - lo.double(), dw.double()
        # third-order terms of moves of 0.05, bf16 gradients, fp32 losses
        size = (grad * step).abs().sum()
        assert abs(float(num - (grad * step).sum())) <= 1e-2 * float(size)


def test_operators_on_a_side_stream_and_in_a_graph():
    T, V, d, E = 96, 1500, 256, 16
    x, w, target = _head_case(T, V, d, 111)
    x, w = x.bfloat16(), w.bfloat16()
    g = torch.full((T,), 1.0 / T, device="cuda")
    gamma = 1.0 + 0.1 * _randn(115, d)
    logits, idx = _randn(116, T, E), _selected(T, E, 2, 117)
    head = eat.EatHead(w, T, grad=True)

    def step():
        y, h = eat.rms_norm(x, gamma, EPS, residual=x)
        nll, lse, dy, dw = head.nll_grad(y, target, g)
        dx, dgamma = eat.rms_norm_grad(h, gamma, EPS, dy)
        loss, counts, n = eat.balance_loss(logits, idx)
        return [nll, lse, dw, dx, dgamma, loss, eat.balance_grad(logits, counts, n, loss)]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_head_refuses_at_call():
    w = torch.zeros(100, 64, dtype=torch.bfloat16, device="cuda")
    head = eat.EatHead(w, 8)
    x = torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(9, dtype=torch.int32, device="cuda")
    with pytest.raises(eat.EatError):
        head.nll(x, t)                      # more than max_tokens
    with pytest.raises(eat.EatError):
        head.nll(x[:0], t[:0])              # none
    with pytest.raises(eat.EatError):
        head.nll_grad(x[:4], t[:4], torch.ones(4, device="cuda"))  # no gradient workspace
    with pytest.raises(ValueError):
        head.nll(x[:4].float(), t[:4])
    with pytest.raises(ValueError):
        head.nll(x[:4], t[:4].long())
    assert head.nll(x[:8], t[:8])[0].isfinite().all()
