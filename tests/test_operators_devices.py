"""The operators on torch tensors: tensors of another device are refused on the host, and a head is made on
its matrix's device.  Fake tensors stand for those of two GPUs; nothing reads them."""
import contextlib

import pytest
import torch

fake = pytest.importorskip("torch._subclasses.fake_tensor")

from paper_2609_33614_gb300 import build, eat  # noqa: E402


@pytest.fixture(scope="module")
def tensors():
    build.build()
    with fake.FakeTensorMode():
        def make(device):
            e = lambda t, *shape: torch.empty(*shape, dtype=t, device=device)
            f, i, b = torch.float32, torch.int32, torch.bfloat16
            return dict(x=e(f, 4, 64), gamma=e(f, 64), logits=e(f, 4, 8), idx=e(i, 4, 2),
                        mask=e(torch.bool, 4), counts=e(i, 8), n=e(i, 1), one=e(f, 1),
                        w=e(b, 100, 64), hx=e(b, 4, 64), target=e(i, 4), g=e(f, 4),
                        w8=e(torch.float8_e4m3fn, 100, 64), x8=e(torch.float8_e4m3fn, 4, 64),
                        s8=e(f, 100), xs=e(f, 4))
        return make("cuda:0"), make("cuda:1")


CALLS = {
    "norm": (lambda o, a: o.norm(a["x"], a["gamma"], 1e-6, None, False), ["gamma"]),
    "norm_residual": (lambda o, a: o.norm(a["x"], a["gamma"], 1e-6, a["residual"], True),
                      ["residual"]),
    "norm_grad": (lambda o, a: o.norm_grad(a["x"], a["gamma"], 1e-6, a["dy"], None),
                  ["gamma", "dy"]),
    "norm_grad_dres": (lambda o, a: o.norm_grad(a["x"], a["gamma"], 1e-6, a["dy"], a["dres"]),
                       ["dres"]),
    "balance_loss": (lambda o, a: o.balance_loss(a["logits"], a["idx"], a["mask"]),
                     ["idx", "mask"]),
    "balance_grad": (lambda o, a: o.balance_grad(a["logits"], a["counts"], a["n"], a["one"],
                                                 a["mask"]), ["counts", "n", "one", "mask"]),
    "head_nll": (lambda o, a: o.head_nll(4096, a["w"], a["hx"], a["target"], None),
                 ["hx", "target"]),
    "head_nll_e4m3": (lambda o, a: o.head_nll(4096, a["w8"], a["x8"], a["target"], a["xs"]),
                      ["x8", "target", "xs"]),
    "head_nll_grad": (lambda o, a: o.head_nll_grad(4096, a["w"], a["hx"], a["target"], a["g"]),
                      ["hx", "target", "g"]),
}


@pytest.mark.parametrize("call,arg", [(c, a) for c, (_, args) in CALLS.items() for a in args])
def test_a_tensor_of_another_device_is_refused(tensors, call, arg):
    near, far = ({**t, "residual": t["x"], "dy": t["x"], "dres": t["x"]} for t in tensors)
    with pytest.raises(ValueError, match="need a tensor on cuda:0, got one on cuda:1"):
        CALLS[call][0](eat._ops(), {**near, arg: far[arg]})


def test_a_head_is_made_on_its_matrix_device(tensors, monkeypatch):
    near, far = tensors
    current, made = ["cuda:0"], []

    @contextlib.contextmanager
    def device(d):
        old, current[0] = current[0], str(d)
        yield
        current[0] = old

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(eat, "_ptr", lambda t: None if t is None else 4096)
    monkeypatch.setattr(eat, "eat_head_create", lambda desc: made.append(current[0]))
    eat.EatHead(near["w"], 4)
    eat.EatHead(far["w"], 4)
    eat.EatHead(far["w8"], 4, w_scale=far["s8"])
    assert made == ["cuda:0", "cuda:1", "cuda:1"] and current == ["cuda:0"]
    with pytest.raises(ValueError, match="need a tensor on cuda:1, got one on cuda:0"):
        eat.EatHead(far["w8"], 4, w_scale=near["s8"])
    assert len(made) == 3
