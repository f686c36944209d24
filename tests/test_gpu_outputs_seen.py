"""GPU: outputs of the calls on torch tensors are torch's to see: dispatch modes, deterministic algorithms, the
profiler and inference mode."""
import contextlib

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2609_33614_gb300 import eat

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_33614_gb300 import build
    build.build()
    torch.cuda.set_device(0)


class Seen(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.shapes = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format:
            self.shapes.append((tuple(out.shape), out.dtype))
        return out


def _x(*shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16)


def _calls():
    x, idx = _x(70, 144), torch.arange(140, device="cuda", dtype=torch.int32).view(70, 2) % 5
    gamma = torch.ones(144, device="cuda")
    logits = torch.randn(70, 5, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    offsets, slot = eat.expert_sort(idx, 5)
    w = torch.rand(70, 2, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    rows = eat.expert_gather(x, slot, offsets)
    xq, xs = eat.quant_rows(x)
    wq, ws = eat.quant_tiles(_x(64, 144))
    return {
        "rms_norm": lambda: eat.rms_norm_fp8(x, gamma, residual=x),
        "rms_norm_grad": lambda: eat.rms_norm_grad(x, gamma, 1e-6, x),
        "balance_loss": lambda: eat.balance_loss(logits, idx),
        "expert_sort": lambda: eat.expert_sort(idx, 5),
        "expert_gather": lambda: eat.expert_gather_fp8(x, slot, offsets),
        "expert_combine_grad": lambda: eat.expert_combine_grad(x, rows, slot, offsets, w),
        "quant_rows": lambda: eat.quant_rows(x),
        "block_mm": lambda: (eat.block_mm(xq, xs, wq, ws),),
        "swiglu": lambda: eat.swiglu_fp8(x),
    }


CALLS = ["rms_norm", "rms_norm_grad", "balance_loss", "expert_sort", "expert_gather", "expert_combine_grad",
         "quant_rows", "block_mm", "swiglu"]


@contextlib.contextmanager
def _deterministic():
    before = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        yield
    finally:
        torch.use_deterministic_algorithms(before)


@pytest.mark.parametrize("name", CALLS)
def test_a_dispatch_mode_sees_them(name):
    call = _calls()[name]
    want = call()
    with Seen() as seen:
        got = call()
    for t, u in zip(got, want):
        assert (tuple(t.shape), t.dtype) in seen.shapes
        assert torch.equal(t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t,
                           u.view(torch.uint8) if u.dtype == torch.float8_e4m3fn else u)


def test_a_mode_that_makes_calls_itself_sees_the_rest():
    x = _x(70, 144)

    class Calls(Seen):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            out = super().__torch_dispatch__(func, types, args, kwargs)
            eat.quant_rows(x)  # (the mode is off within itself)
            return out

    with Calls() as seen:
        outs = eat.quant_rows_columns(x)
    assert len(seen.shapes) == len(outs) == 4


@pytest.mark.parametrize("name", CALLS)
def test_the_profiler_sees_them(name):
    call = _calls()[name]
    call()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as p:
        out = call()
    assert sum(e.name == "aten::empty" for e in p.events()) >= len(out)


def test_deterministic_algorithms_fill_what_no_kernel_writes():
    """The rows and blocks behind the experts' last ones in quant_columns' outputs."""
    x, offsets = _x(300, 64), torch.tensor([0, 40, 40, 100], device="cuda", dtype=torch.int32)
    with _deterministic():
        cq, cscale = eat.quant_columns(x, offsets)
    plain = eat.quant_columns(x, offsets)
    assert len(cq) > 128 and len(cscale) > 2  # experts of 40 and 60 rows: 64 + 64 rows, two blocks
    assert cq[128:].float().isnan().all() and cscale[2:].isnan().all()
    assert torch.equal(cq[:128].view(torch.uint8), plain[0][:128].view(torch.uint8))
    assert torch.equal(cscale[:2], plain[1][:2])


def test_inference_mode_makes_inference_tensors():
    x = _x(9, 64)
    with torch.inference_mode():
        q, scale = eat.quant_rows(x)
    assert q.is_inference() and scale.is_inference()
    assert not eat.quant_rows(x)[0].is_inference()
