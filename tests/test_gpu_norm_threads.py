"""GPU: the norm's gradient from several host threads."""
import threading

import pytest
import torch

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def test_gradients_of_different_widths_from_two_threads():
    """Calls of one kernel with different amounts of shared memory, from host threads of their own (the
    ctypes calls run without Python's lock)."""
    T, calls, failed, alone = 1300, 4000, [], {}
    cases = []
    for k, d in enumerate((2048, 4096)):
        gen = torch.Generator("cuda").manual_seed(k)
        h, dy = (torch.randn(T, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        gamma = 1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")
        work = torch.empty(eat.eat_rms_norm_grad_workspace(T, d), dtype=torch.uint8, device="cuda")
        alone[d] = eat.rms_norm_grad(h, gamma, EPS, dy)
        cases.append((d, h, gamma, dy, torch.empty_like(h), torch.empty(d, device="cuda"), work,
                      torch.cuda.Stream()))
    torch.cuda.synchronize()
    f = eat.lib().eat_rms_norm_grad
    start = threading.Barrier(2)

    def loop(d, h, gamma, dy, dx, dgamma, work, stream):
        args = (h.data_ptr(), T, d, eat.EAT_BF16, gamma.data_ptr(), EPS, dy.data_ptr(), None,
                dx.data_ptr(), dgamma.data_ptr(), work.data_ptr(), stream.cuda_stream)
        start.wait()
        for _ in range(calls):
            s = f(*args)
            if s != eat.EAT_OK:
                failed.append((d, s))
                return

    threads = [threading.Thread(target=loop, args=c) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for d, _, _, _, dx, dgamma, _, _ in cases:
        assert torch.equal(dx, alone[d][0]) and torch.equal(dgamma, alone[d][1])
