"""GPU: gradients that would be written over what their call reads are refused (before any launch)."""
import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

T, V, D = 6, 40, 64


@pytest.mark.parametrize("dx,dw,word", [
    ("x", "free", "dx"), ("x+16", "free", "dx"), ("x-16", "free", "dx"), ("w", "free", "dx"),
    ("w+80", "free", "dx"), ("out", "w", "dw"), ("out", "w+16", "dw"), ("out", "w-16", "dw"),
    ("out", "x", "dw"), ("free", "free", "dw"), ("free+16", "free", "dw"), ("out", "free", None)])
def test_overlapping_gradients_are_refused(dx, dw, word):
    from paper_2609_33614_gb300 import build
    build.build()
    gen = torch.Generator("cuda").manual_seed(1)
    # x, w, out and free, 64 KB apart in one buffer, so that every shifted address is the test's own
    buf = torch.randn(4, 32768, generator=gen, device="cuda").bfloat16()
    at = {n: buf[i, 4096:].data_ptr() for i, n in enumerate(("x", "w", "out", "free"))}
    x, w = buf[0, 4096:4096 + T * D].view(T, D), buf[1, 4096:4096 + V * D].view(V, D)
    y = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    g, nll = torch.ones(T, device="cuda"), torch.empty(T, device="cuda")
    head = eat.EatHead(w, T, grad=True)

    def address(s):
        for sign in "+-":
            if sign in s:
                name, n = s.split(sign)
                return at[name] + int(sign + n)
        return at[s]

    torch.cuda.synchronize()
    before = buf.clone()
    status = eat.lib().eat_head_nll_grad(head.h, x.data_ptr(), T, y.data_ptr(), g.data_ptr(),
                                         nll.data_ptr(), None, address(dx), address(dw),
                                         torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    if word is None:
        assert status == eat.EAT_OK
        want = head.nll_grad(x, y, g)
        assert torch.equal(buf[2, 4096:4096 + T * D].view(T, D), want[2])
        assert torch.equal(buf[3, 4096:4096 + V * D].view(V, D), want[3])
        assert torch.equal(buf[:2], before[:2])
    else:
        assert status == eat.EAT_ERR_INVALID_ARG
        assert f"{word} must not overlap" in eat.lib().eat_last_error(None).decode()
        assert torch.equal(buf, before)
    head.close()
