"""The vocabulary head's failure state, and its handles beside one another."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def _case(T, V, d, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    w = 0.05 * torch.randn(V, d, generator=g, device="cuda")
    x = torch.randn(T, d, generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    return x.bfloat16(), w.bfloat16(), y


@pytest.mark.parametrize("T", [5, 60, 300])
@pytest.mark.parametrize("grad", [False, True])
def test_expired_wait_is_reported_and_reset(T, grad):
    """A wait that gave up (host-made: nothing arrives on its barrier): NaN results, then
    EAT_ERR_STATE until the reset."""
    x, w, y = _case(T, 700, 128, 5)
    g = torch.ones(T, device="cuda")
    head = eat.EatHead(w, T, grad=True)
    call = lambda: head.nll_grad(x, y, g) if grad else head.nll(x, y)
    want = call()
    eat.eat_head_selftest_expire_wait(head.h, 10_000)
    got = call()
    torch.cuda.synchronize()
    assert all(t.isnan().all() for t in (got[:3] if grad else got))
    for _ in range(2):
        with pytest.raises(eat.EatError) as ei:
            call()
        assert ei.value.status == eat.EAT_ERR_STATE
    eat.eat_head_reset(head.h)
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    with pytest.raises(eat.EatError):
        eat.eat_head_selftest_expire_wait(head.h, 10)
    head.close()


def test_heads_on_two_streams():
    """Calls of two handles may overlap; each gives what it gives alone."""
    heads, args, want = [], [], []
    for k, (T, V, d) in enumerate(((64, 9000, 256), (200, 5000, 512))):
        x, w, y = _case(T, V, d, 11 + k)
        g = torch.full((T,), 1.0 / T, device="cuda")
        heads.append(eat.EatHead(w, T, grad=True))
        args.append((x, y, g))
        want.append((heads[k].nll(x, y), heads[k].nll_grad(x, y, g)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in heads]
    got = [[], []]
    for _ in range(6):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append((heads[k].nll(*args[k][:2]), heads[k].nll_grad(*args[k])))
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in got[k]:
            assert all(torch.equal(u, v) for u, v in zip(a + b, want[k][0] + want[k][1]))


def test_vocabulary_updated_in_place():
    """w may change between calls, in stream order."""
    x, w, y = _case(40, 3000, 256, 21)
    head = eat.EatHead(w, 40)
    a = head.nll(x, y)[0].clone()
    w.mul_(2.0)
    b = head.nll(x, y)[0]
    assert not torch.equal(a, b)
    assert torch.equal(eat.EatHead(w.clone(), 40).nll(x, y)[0], b)


@pytest.mark.parametrize("T,times", [(1, 1.3), (4, 1.3), (32, 1.3), (33, 1.3), (64, 1.3), (65, 1.3),
                                     (128, 1.3), (129, 1.9), (700, 1.9)])
def test_gradients_are_little_more_than_rounded_once(T, times):
    """The error of dx and dw beside that of rounding the exact gradients to bf16 once.  dx's target
    terms are exact, and dw's with up to 128 tokens; with more they carry one rounding of their own
    (1.41 where both are as large on average; mantissas shift it)."""
    x, w, y = _case(T, 6000, 256, 31)
    g = torch.rand(T, generator=torch.Generator("cuda").manual_seed(5), device="cuda") / T
    _, _, dx, dw = eat.EatHead(w, T, grad=True).nll_grad(x, y, g)
    x64, w64 = x.double(), w.double()
    p = torch.softmax(x64 @ w64.T, 1)
    p[torch.arange(T, device="cuda"), y.long()] -= 1.0
    p *= g.double()[:, None]
    for got, want, k in ((dx, p @ w64, 1.3), (dw, p.T @ x64, times)):
        once = (want.bfloat16().double() - want).norm()
        assert (got.double() - want).norm() <= k * once


@pytest.mark.parametrize("ignored", [0.1, 0.6, 0.97])
def test_gradient_in_pieces_of_tokens(ignored):
    """A vocabulary of 2^20 rows takes 256 tokens at a time (512 MB of exponentials): sums of dw that
    go on over pieces, a last piece with few tokens, pieces without any."""
    T, V, d = 700, 1 << 20, 64
    x, w, y = _case(T, V, d, 41)
    gen = torch.Generator("cuda").manual_seed(42)
    drop = torch.rand(T, generator=gen, device="cuda") < ignored
    x[drop] = float("nan")
    y = torch.where(drop, -1, y)
    g = torch.rand(T, generator=gen, device="cuda") / T
    head = eat.EatHead(w, T, grad=True)
    nll, lse, dx, dw = head.nll_grad(x, y, g)
    on = ~drop
    x64, w64 = x[on].double(), w.double()
    logits = x64 @ w64.T
    want = torch.logsumexp(logits, 1)
    assert ((lse[on].double() - want).abs() <= 1e-5 * want.abs()).all()
    p = logits.sub_(want[:, None]).exp_()
    p[torch.arange(int(on.sum()), device="cuda"), y[on].long()] -= 1.0
    p *= g[on].double()[:, None]
    ref = p @ w64
    assert (dx[on].double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    assert (dx[drop] == 0).all() and (nll[drop] == 0).all()
    ref = p.T @ x64
    del p, logits
    assert (dw.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    head.close()
