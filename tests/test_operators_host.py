"""The operators around the layer (norm, balance loss, vocabulary head): what they refuse on the host,
before any device work."""
import ctypes

import pytest
import torch

from paper_2609_33614_gb300 import build, eat

A = [4096 * i for i in range(1, 12)]  # aligned stand-ins: no address is read


@pytest.fixture(scope="module")
def lib():
    build.build()
    return eat.lib()


def _refuses(lib, r, status, word):
    assert r == status, lib.eat_last_error(None)
    assert word in lib.eat_last_error(None).decode()


NORM = dict(x=A[0], residual=None, T=4, d=64, xdtype=eat.EAT_BF16, gamma=A[1], eps=1e-6, h=None,
            y=A[2], ydtype=eat.EAT_BF16, y_scale=None, stream=None)


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "non-NULL"), (dict(gamma=None), "non-NULL"), (dict(y=None), "non-NULL"),
    (dict(residual=A[3]), "residual needs h"), (dict(T=0), "T >= 1"), (dict(T=-1), "T >= 1"),
    (dict(d=0), "d <= 65536"), (dict(d=65537), "d <= 65536"),
    (dict(xdtype=eat.EAT_FP8_E4M3), "xdtype"), (dict(xdtype=7), "xdtype"),
    (dict(ydtype=eat.EAT_F32), "ydtype"), (dict(ydtype=eat.EAT_FP8_E4M3), "y_scale"),
    (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(x=A[0] + 1), "misaligned"),
    (dict(gamma=A[1] + 2), "misaligned"), (dict(y=A[2] + 1), "misaligned"),
    (dict(residual=A[3], h=A[4] + 1), "misaligned"),
    (dict(ydtype=eat.EAT_FP8_E4M3, y_scale=A[5] + 2), "misaligned"),
])
def test_rms_norm_refuses(lib, kw, word):
    _refuses(lib, lib.eat_rms_norm(*{**NORM, **kw}.values()), eat.EAT_ERR_INVALID_ARG, word)


GRAD = dict(h=A[0], T=4, d=64, xdtype=eat.EAT_F32, gamma=A[1], eps=1e-6, dy=A[2], dres=None,
            dx=A[3], dgamma=A[4], work=A[5], stream=None)


@pytest.mark.parametrize("kw,word", [
    (dict(h=None), "non-NULL"), (dict(dy=None), "non-NULL"), (dict(dx=None), "non-NULL"),
    (dict(dgamma=None), "non-NULL"), (dict(work=None), "non-NULL"), (dict(T=0), "T >= 1"),
    (dict(d=70000), "d <= 65536"), (dict(xdtype=2), "xdtype"), (dict(eps=0.0), "eps"),
    (dict(dres=A[6] + 2), "misaligned"), (dict(work=A[5] + 8), "misaligned"),
])
def test_rms_norm_grad_refuses(lib, kw, word):
    _refuses(lib, lib.eat_rms_norm_grad(*{**GRAD, **kw}.values()), eat.EAT_ERR_INVALID_ARG, word)


LOSS = dict(logits=A[0], T=4, E=8, K=2, idx=A[1], mask=None, loss=A[2], counts=A[3], n=A[4],
            work=A[5], stream=None)
BGRAD = dict(logits=A[0], T=4, E=8, mask=None, counts=A[1], n=A[2], g=A[3], dlogits=A[4],
             stream=None)


@pytest.mark.parametrize("kw,word", [
    (dict(logits=None), "non-NULL"), (dict(idx=None), "non-NULL"), (dict(work=None), "non-NULL"),
    (dict(T=0), "T >= 1"), (dict(E=0), "E <= 256"), (dict(E=257), "E <= 256"),
    (dict(K=0), "K <= 16"), (dict(K=17), "K <= 16"), (dict(idx=A[1] + 1), "misaligned"),
])
def test_balance_loss_refuses(lib, kw, word):
    _refuses(lib, lib.eat_balance_loss(*{**LOSS, **kw}.values()), eat.EAT_ERR_INVALID_ARG, word)


@pytest.mark.parametrize("kw,word", [
    (dict(logits=None), "non-NULL"), (dict(g=None), "non-NULL"), (dict(counts=None), "non-NULL"),
    (dict(T=0), "T >= 1"), (dict(E=257), "E <= 256"), (dict(dlogits=A[4] + 2), "misaligned"),
])
def test_balance_grad_refuses(lib, kw, word):
    _refuses(lib, lib.eat_balance_grad(*{**BGRAD, **kw}.values()), eat.EAT_ERR_INVALID_ARG, word)


def test_workspaces_are_bounded(lib):
    assert lib.eat_rms_norm_grad_workspace(0, 64) == 0
    assert lib.eat_balance_workspace(0, 8) == 0
    for T in (1, 7, 4096, 1 << 30):
        assert 0 < lib.eat_rms_norm_grad_workspace(T, 65536) <= 1 << 30
        assert 0 < lib.eat_balance_workspace(T, 256) <= 1 << 22


HEAD = dict(d_model=256, vocab=1000, max_tokens=64, dtype=eat.EAT_BF16, with_grad=0, w=A[0],
            w_scale=None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=eat.EAT_F32), eat.EAT_ERR_UNSUPPORTED, "dtype"),
    (dict(dtype=9), eat.EAT_ERR_UNSUPPORTED, "dtype"),
    (dict(d_model=0), eat.EAT_ERR_UNSUPPORTED, "d_model"),
    (dict(d_model=100), eat.EAT_ERR_UNSUPPORTED, "d_model"),
    (dict(d_model=16448), eat.EAT_ERR_UNSUPPORTED, "d_model"),
    (dict(vocab=0), eat.EAT_ERR_UNSUPPORTED, "vocab"),
    (dict(vocab=(1 << 20) + 1), eat.EAT_ERR_UNSUPPORTED, "vocab"),
    (dict(max_tokens=0), eat.EAT_ERR_INVALID_ARG, "max_tokens"),
    (dict(max_tokens=65537), eat.EAT_ERR_INVALID_ARG, "max_tokens"),
    (dict(w=None), eat.EAT_ERR_INVALID_ARG, "w is NULL"),
    (dict(w=A[0] + 8), eat.EAT_ERR_INVALID_ARG, "aligned"),
    (dict(dtype=eat.EAT_FP8_E4M3), eat.EAT_ERR_INVALID_ARG, "w_scale"),
    (dict(dtype=eat.EAT_FP8_E4M3, w_scale=A[1], with_grad=1), eat.EAT_ERR_UNSUPPORTED, "BF16"),
])
def test_head_create_refuses(lib, kw, status, word):
    h = ctypes.c_void_p(1234)
    desc = eat.eat_head_desc(*{**HEAD, **kw}.values())
    _refuses(lib, lib.eat_head_create(ctypes.byref(desc), ctypes.byref(h)), status, word)
    assert h.value is None


def test_head_null_calls(lib):
    assert lib.eat_head_create(None, None) == eat.EAT_ERR_INVALID_ARG
    assert lib.eat_head_nll(None, 16, None, 1, 16, 16, None, None) == eat.EAT_ERR_INVALID_ARG
    assert lib.eat_head_nll_grad(None, 16, 1, 16, 16, 16, None, 16, 16, None) == \
        eat.EAT_ERR_INVALID_ARG
    assert lib.eat_head_reset(None, None) == eat.EAT_ERR_INVALID_ARG
    assert lib.eat_head_destroy(None) == eat.EAT_OK


def test_wrappers_check_tensors():
    """CPU tensors, other shapes or types never reach the library."""
    x, g = torch.zeros(4, 64), torch.ones(64)
    for call in (lambda: eat.rms_norm(x, g), lambda: eat.rms_norm(x.to(torch.float16), g),
                 lambda: eat.rms_norm_fp8(x[0], g), lambda: eat.rms_norm_grad(x, g, 1e-6, x),
                 lambda: eat.balance_loss(x, torch.zeros(4, 2, dtype=torch.int64)),
                 lambda: eat.EatHead(x, 4)):
        with pytest.raises(ValueError):
            call()
