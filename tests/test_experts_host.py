"""Rows sorted by expert, their e4m3 products and the gated activation: what is refused on the host, before
any device work."""
import pytest
import torch

from paper_2609_33614_gb300 import build, eat

A = [4096 * i for i in range(1, 12)]  # aligned stand-ins: no address is read
F32, BF16, FP8 = eat.EAT_F32, eat.EAT_BF16, eat.EAT_FP8_E4M3
BAD = eat.EAT_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    build.build()
    return eat.lib()


SORT = dict(idx=A[0], T=4, K=2, E=8, mask=None, offsets=A[1], slot=A[2], work=A[3], stream=None)
GATHER = dict(x=A[0], T=4, K=2, E=8, d=64, dtype=BF16, slot=A[1], offsets=A[2], rows=A[3],
              rows_dtype=BF16, scale=None, stream=None)
COMBINE = dict(rows=1 << 20, T=4, K=2, d=64, dtype=F32, slot=A[1], w=None, y=1 << 21, stream=None)
CGRAD = dict(dy=1 << 20, rows=1 << 21, T=4, K=2, E=8, d=64, dtype=BF16, slot=A[0], offsets=A[1],
             w=A[2], drows=1 << 22, dw=A[3], stream=None)
QROWS = dict(x=A[0], M=4, K=64, dtype=BF16, q=A[1], scale=A[2], stream=None)
QCOLS = dict(x=A[0], M=4, K=64, dtype=BF16, offsets=A[1], E=2, q=A[2], scale=A[3], cq=A[4],
             cscale=A[5], stream=None)
QTILES = dict(w=1 << 20, E=2, N=64, K=64, dtype=F32, q=1 << 21, scale=A[2], stream=None)
MM = dict(xq=1 << 20, xs=A[0], wq=1 << 21, ws=A[1], offsets=A[2], E=2, M=4, N=64, K=64, transposed=0,
          y=1 << 22, ydtype=BF16, stream=None)
MGRAD = dict(gq=1 << 20, gs=A[0], xq=1 << 21, xs=A[1], offsets=A[2], E=2, rows=64, blocks=2, N=64,
             K=64, dw=1 << 22, dtype=BF16, stream=None)
GLU = dict(gu=A[0], R=4, F=64, dtype=BF16, h=A[1], h_dtype=BF16, scale=None, stream=None)
GLUGRAD = dict(gu=A[0], dh=A[1], R=4, F=64, dtype=BF16, dgu=A[2], stream=None)
UNS = eat.EAT_ERR_UNSUPPORTED

CASES = [
    ("eat_expert_sort", SORT, [
        (dict(idx=None), "non-NULL"), (dict(T=1 << 20, work=None), "needs work"), (dict(T=0), "T >= 1"),
        (dict(K=0), "K <= 16"), (dict(K=17), "K <= 16"), (dict(T=1 << 30, K=2), "2^30"),
        (dict(E=0), "E <= 256"), (dict(E=257), "E <= 256"), (dict(idx=A[0] + 2), "misaligned"),
        (dict(work=A[3] + 4), "misaligned")]),
    ("eat_expert_gather", GATHER, [
        (dict(slot=None), "non-NULL"), (dict(rows=None), "non-NULL"), (dict(d=0), "d <= 65536"),
        (dict(d=65537), "d <= 65536"), (dict(dtype=FP8), "dtype"), (dict(rows_dtype=F32), "rows_dtype"),
        (dict(rows_dtype=FP8), "scale"), (dict(x=A[0] + 1), "misaligned"),
        (dict(rows_dtype=FP8, scale=A[4] + 2), "misaligned"), (dict(rows=A[0] + 256), "overlaps")]),
    ("eat_expert_combine", COMBINE, [
        (dict(y=None), "non-NULL"), (dict(T=-1), "T >= 1"), (dict(w=A[2] + 1), "misaligned"),
        (dict(y=(1 << 20) + 1024), "overlaps"), (dict(dtype=5), "dtype")]),
    ("eat_expert_combine_grad", CGRAD, [
        (dict(w=None), "non-NULL"), (dict(dw=None), "non-NULL"), (dict(drows=(1 << 21) + 64), "overlaps"),
        (dict(drows=1 << 20), "overlaps"), (dict(E=300), "E <= 256")]),
    ("eat_quant_rows", QROWS, [
        (dict(q=None), "non-NULL"), (dict(M=0), "rows"), (dict(M=(1 << 30) + 1), "rows"),
        (dict(K=0), "columns"), (dict(K=65537), "columns"), (dict(dtype=FP8), "dtype"),
        (dict(x=A[0] + 1), "misaligned"), (dict(scale=A[2] + 2), "misaligned"),
        (dict(q=A[0] + 504), "overlaps")]),
    ("eat_quant_columns", QCOLS, [
        (dict(q=A[0] + 16), "overlaps"), (dict(cq=A[0] - 128), "overlaps"),
        (dict(cq=None), "non-NULL"), (dict(scale=None), "together"), (dict(q=None), "together"),
        (dict(E=0), "E <= 256"), (dict(offsets=None), "offsets"), (dict(M=1 << 30), "padded"),
        (dict(offsets=A[1] + 2), "misaligned")]),
    ("eat_quant_tiles", QTILES, [
        (dict(w=None), "non-NULL"), (dict(N=0), "N <= 65536"), (dict(E=257), "E <= 256"),
        (dict(w=(1 << 20) + 2), "misaligned"), (dict(q=(1 << 20) + 32), "overlaps")]),
    ("eat_block_mm", MM, [
        (dict(y=(1 << 20) + 32), "overlaps"), (dict(y=(1 << 21) - 64), "overlaps"),
        (dict(xs=None), "non-NULL"), (dict(y=None), "non-NULL"), (dict(M=0), "rows"),
        (dict(N=0), "N and K"), (dict(K=65537), "N and K"), (dict(offsets=None), "offsets"),
        (dict(ydtype=FP8), "dtype"), (dict(xq=(1 << 20) + 8), "misaligned"),
        (dict(wq=(1 << 21) + 4), "misaligned"), (dict(y=(1 << 22) + 1), "misaligned")]),
    ("eat_block_mm_grad", MGRAD, [
        (dict(gs=None), "non-NULL"), (dict(rows=0), "rows"), (dict(blocks=0), "blocks"),
        (dict(offsets=None), "offsets"), (dict(dtype=FP8), "dtype"),
        (dict(xq=(1 << 21) + 8), "misaligned"), (dict(dw=(1 << 20) + 64), "overlaps"),
        (dict(dw=1 << 21), "overlaps")]),
    ("eat_swiglu", GLU, [
        (dict(h=None), "non-NULL"), (dict(F=0), "columns"), (dict(R=0), "rows"),
        (dict(h_dtype=F32), "h_dtype"), (dict(h_dtype=FP8), "scale"), (dict(gu=A[0] + 1), "misaligned"),
        (dict(h=A[0] + 512), "overlaps")]),
    ("eat_swiglu_grad", GLUGRAD, [
        (dict(dh=None), "non-NULL"), (dict(dtype=FP8), "dtype"), (dict(dgu=A[2] + 1), "misaligned"),
        (dict(dgu=A[1] - 64), "overlaps"), (dict(dgu=A[0] + 16), "overlaps")]),
]


@pytest.mark.parametrize("fn,base,kw,word", [(f, b, k, w) for f, b, cs in CASES for k, w in cs])
def test_refuses(lib, fn, base, kw, word):
    r = getattr(lib, fn)(*{**base, **kw}.values())
    text = lib.eat_last_error(None).decode()
    assert r == BAD and text.startswith(fn) and word in text, text


@pytest.mark.parametrize("fn,base,kw", [
    ("eat_block_mm", MM, dict(K=72)), ("eat_block_mm", MM, dict(N=72, transposed=1)),
    ("eat_block_mm_grad", MGRAD, dict(N=8)), ("eat_block_mm_grad", MGRAD, dict(K=100))])
def test_widths_that_are_not_supported(lib, fn, base, kw):
    assert getattr(lib, fn)(*{**base, **kw}.values()) == UNS
    assert "multiples of 16" in lib.eat_last_error(None).decode()


def test_workspaces_and_padded_sizes(lib):
    assert lib.eat_expert_sort_workspace(16384, 8, 64) == 0 < lib.eat_expert_sort_workspace(16385, 8, 64)
    assert lib.eat_expert_sort_workspace(0, 8, 64) == 0 == lib.eat_expert_sort_workspace(1 << 20, 17, 64)
    rows, blocks = lib.eat_quant_columns_rows, lib.eat_quant_columns_blocks
    assert (rows(1, 1), rows(32, 1), rows(33, 1), rows(2, 64)) == (32, 32, 64, 64)
    assert (blocks(1, 1), blocks(128, 1), blocks(129, 1), blocks(2, 64)) == (1, 1, 2, 2)
    assert rows(0, 1) == 0 == blocks(5, 257)
    g = torch.Generator().manual_seed(1)
    for E in (1, 2, 7, 64, 256):  # enough for every split
        for top in (1, 2, 40, 300):
            n = torch.randint(0, top + 1, (E,), generator=g)
            M = int(n.sum())
            if M:
                assert rows(M, E) >= int(((n + 31) // 32 * 32).sum())
                assert blocks(M, E) >= int(((n + 127) // 128).sum())
                assert blocks(M, E) * 128 >= rows(M, E)


# ------------------------------------------------------------------- tensors (fake ones of two GPUs)
fake = pytest.importorskip("torch._subclasses.fake_tensor")


@pytest.fixture(scope="module")
def tensors(lib):
    with fake.FakeTensorMode():
        def make(device):
            e = lambda t, *shape: torch.empty(*shape, dtype=t, device=device)
            f, i, b, q = torch.float32, torch.int32, torch.bfloat16, torch.float8_e4m3fn
            return dict(idx=e(i, 4, 2), mask=e(torch.bool, 4), x=e(b, 4, 64), slot=e(i, 4, 2),
                        offsets=e(i, 3), rows=e(b, 8, 64), w=e(f, 4, 2), dy=e(b, 4, 64),
                        weights=e(b, 2, 32, 64), xq=e(q, 8, 64), xs=e(f, 1, 8), wq=e(q, 2, 32, 64),
                        ws=e(f, 2, 1, 1), cq=e(q, 64, 64), cs=e(f, 2, 64), gq=e(q, 64, 32),
                        gs=e(f, 2, 32), gu=e(b, 4, 128), dh=e(b, 4, 64))
        return make("cuda:0"), make("cuda:1")


CALLS = {
    "expert_sort": (lambda o, a: o.expert_sort(a["idx"], 8, a["mask"]), ["mask"]),
    "expert_gather": (lambda o, a: o.expert_gather(a["x"], a["slot"], a["offsets"], False),
                      ["slot", "offsets"]),
    "expert_combine": (lambda o, a: o.expert_combine(a["rows"], a["slot"], a["w"]), ["slot", "w"]),
    "expert_combine_grad": (lambda o, a: o.expert_combine_grad(a["dy"], a["rows"], a["slot"],
                                                               a["offsets"], a["w"]),
                            ["rows", "slot", "offsets", "w"]),
    "quant_columns": (lambda o, a: o.quant_columns(a["rows"], a["offsets"], True), ["offsets"]),
    "block_mm": (lambda o, a: o.block_mm(a["xq"], a["xs"], a["wq"], a["ws"], a["offsets"], False, None),
                 ["xs", "wq", "ws", "offsets"]),
    "block_mm_grad": (lambda o, a: o.block_mm_grad(a["gq"], a["gs"], a["cq"], a["cs"], a["offsets"],
                                                   None), ["gs", "cq", "cs", "offsets"]),
    "swiglu_grad": (lambda o, a: o.swiglu_grad(a["gu"], a["dh"]), ["dh"]),
}


@pytest.mark.parametrize("call,arg", [(c, a) for c, (_, args) in CALLS.items() for a in args])
def test_a_tensor_of_another_device_is_refused(tensors, call, arg):
    near, far = tensors
    with pytest.raises(ValueError, match="need a tensor on cuda:0, got one on cuda:1"):
        CALLS[call][0](eat._ops(), {**near, arg: far[arg]})


@pytest.mark.parametrize("call,arg,shape,dtype,word", [
    ("expert_sort", "idx", (4, 2), torch.int64, "idx"), ("expert_sort", "idx", (8,), torch.int32, "matrix"),
    ("expert_sort", "mask", (5,), torch.bool, "mask"),
    ("expert_gather", "slot", (5, 2), torch.int32, "slot"),
    ("expert_gather", "x", (4, 64), torch.float16, "fp32 or bf16"),
    ("expert_gather", "offsets", (1,), torch.int32, "offsets"),
    ("expert_combine", "rows", (9, 64), torch.bfloat16, "rows"),
    ("expert_combine", "w", (4, 2), torch.bfloat16, "w: need"),
    ("expert_combine_grad", "rows", (8, 64), torch.float32, "rows"),
    ("expert_combine_grad", "dy", (5, 64), torch.bfloat16, "slot"),
    ("block_mm", "xq", (8, 64), torch.bfloat16, "xq"), ("block_mm", "xq", (8, 96), torch.float8_e4m3fn, "xq"),
    ("block_mm", "xs", (8, 1), torch.float32, "xs"), ("block_mm", "wq", (32, 64), torch.float8_e4m3fn, "wq"),
    ("block_mm", "wq", (3, 32, 64), torch.float8_e4m3fn, "wq"), ("block_mm", "ws", (2, 1), torch.float32, "ws"),
    ("block_mm_grad", "gq", (96, 32), torch.float8_e4m3fn, "xq"),
    ("block_mm_grad", "gs", (1, 32), torch.float32, "xs"),
    ("swiglu_grad", "gu", (4, 127), torch.bfloat16, "2 F"), ("swiglu_grad", "dh", (4, 63), torch.bfloat16, "dh"),
])
def test_a_tensor_of_another_shape_or_type_is_refused(tensors, call, arg, shape, dtype, word):
    with fake.FakeTensorMode():
        t = torch.empty(*shape, dtype=dtype, device="cuda:0")
    with pytest.raises(ValueError, match=word):
        CALLS[call][0](eat._ops(), {**tensors[0], arg: t})


def test_tensors_that_are_not_contiguous_or_not_cuda(tensors):
    near, _ = tensors
    with fake.FakeTensorMode():
        rows = torch.empty(8, 128, dtype=torch.bfloat16, device="cuda:0")[:, :64]
    with pytest.raises(ValueError, match="contiguous"):
        eat.expert_combine(rows, near["slot"])
    with pytest.raises(ValueError, match="CUDA"):
        eat.quant_rows(torch.zeros(4, 64))
    with pytest.raises(ValueError, match="torch.bfloat16 or torch.float32"):
        eat._ops().block_mm(*[near[n] for n in ("xq", "xs", "wq", "ws", "offsets")], False, torch.float16)
    with pytest.raises(ValueError, match="without offsets"):
        eat._ops().block_mm(*[near[n] for n in ("xq", "xs", "wq", "ws")], None, False, None)
    with pytest.raises(TypeError):
        eat.expert_sort(near["idx"], None)
