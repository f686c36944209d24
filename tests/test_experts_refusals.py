"""Block-scaled products and sorted rows: calls that the C entry points refuse, host only."""
import pytest

from paper_2609_33614_gb300 import build, eat
from test_experts_host import (A, BF16, CGRAD, COMBINE, F32, FP8, GATHER, GLU, GLUGRAD, MGRAD, MM, QCOLS, QROWS,
                               QTILES, SORT)

BAD = eat.EAT_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    build.build()
    return eat.lib()


def _refused(lib, fn, args, word):
    assert getattr(lib, fn)(*args) == BAD
    text = lib.eat_last_error(None).decode()
    assert text.startswith(fn) and word in text, text


@pytest.mark.parametrize("rows,blocks,word", [
    (100, 1, "multiple of 32"), (1, 1, "multiple of 32"), (33, 8, "multiple of 32"),
    (256, 1, "blocks"), (160, 1, "blocks"), (64, 0, "blocks"), (64, -3, "blocks"), (1 << 30, 7, "blocks")])
@pytest.mark.parametrize("offsets,E", [(None, 1), (1 << 16, 2)])
def test_operands_of_a_weights_gradient_that_are_not_all_there(lib, rows, blocks, word, offsets, E):
    """Rows or blocks that eat_quant_columns_rows and _blocks never give: an expert that reaches beyond them
    would add nothing to dw."""
    _refused(lib, "eat_block_mm_grad",
             {**MGRAD, "rows": rows, "blocks": blocks, "offsets": offsets, "E": E}.values(), word)


def test_every_operand_of_quant_columns_has_the_rows_and_blocks(lib):
    for E in (1, 2, 7, 64, 256):
        for M in list(range(1, 700)) + [4095, 4096, 70001, (1 << 30) - 31 * 256]:
            rows, blocks = lib.eat_quant_columns_rows(M, E), lib.eat_quant_columns_blocks(M, E)
            assert rows % 32 == 0 and blocks >= -(-rows // 128) >= 1


@pytest.mark.parametrize("fn,base", [("eat_block_mm_selftest", MM), ("eat_block_mm_grad_selftest", MGRAD)])
@pytest.mark.parametrize("kw,word", [
    (dict(limit_ns=999_999), "limit_ns"), (dict(limit_ns=10 ** 9 + 1), "limit_ns"), (dict(status=None), "status"),
    (dict(status=A[6] + 2), "status"), (dict(copies=-1), "copies"), (dict(xs=None), "non-NULL"),
    (dict(K=65537), "N and K")])
def test_selftests_of_the_waits(lib, fn, base, kw, word):
    args = {n: v for n, v in base.items() if n != "stream"}
    args.update(limit_ns=10 ** 6, cta=0, copies=1, status=A[6], stream=None)
    _refused(lib, fn, {**args, **kw}.values(), word)


def test_a_null_handle_has_no_limit_of_its_waits(lib):
    _refused(lib, "eat_head_selftest_wait_limit", (None, 10 ** 6), "null handle")


BIG = 1 << 30  # apart from every other stand-in
# the last element of the array that the output's first one lies on, or the other way round
OVERLAPS = [
    ("eat_expert_sort", SORT, [
        dict(offsets=A[0] + 28), dict(slot=A[0] - 28), dict(slot=A[1] + 32), dict(mask=A[2] + 28),
        dict(mask=BIG + 3, offsets=BIG), dict(T=1 << 20, idx=1 << 26, slot=1 << 27, work=(1 << 26) + 16),
        dict(T=1 << 20, idx=1 << 26, slot=1 << 27, work=(1 << 27) + (1 << 23) - 16)]),
    ("eat_expert_gather", GATHER, [
        dict(rows=A[1] + 28), dict(rows=A[2] + 32), dict(rows_dtype=FP8, scale=A[0] + 508),
        dict(rows_dtype=FP8, scale=A[3] + 508), dict(rows_dtype=FP8, scale=A[1] - 28),
        dict(rows_dtype=FP8, scale=A[2] - 28)]),
    ("eat_expert_combine", COMBINE, [dict(y=A[1] + 28), dict(w=(1 << 21) + 1020), dict(y=(1 << 20) + 2044)]),
    ("eat_expert_combine_grad", CGRAD, [
        dict(drows=A[0] + 28), dict(drows=A[1] + 32), dict(drows=A[2] + 28), dict(dw=A[2]), dict(dw=A[0] - 28),
        dict(dw=A[1] + 32), dict(dw=(1 << 22) + 1020), dict(dw=(1 << 20) + 508), dict(dw=(1 << 21) + 1020)]),
    ("eat_quant_rows", QROWS, [dict(scale=A[0] + 508), dict(scale=A[1] + 252), dict(q=A[2] + 15)]),
    ("eat_quant_columns", QCOLS, [
        dict(scale=A[0] + 508), dict(cscale=A[0] + 508), dict(cq=A[1] + 11), dict(q=A[1] + 11),
        dict(scale=A[2] + 252), dict(cscale=A[4] + 4092), dict(cq=A[2] + 255), dict(cscale=A[3] + 12),
        dict(q=None, scale=None, cscale=A[4])]),
    ("eat_quant_tiles", QTILES, [dict(scale=(1 << 20) + 32764), dict(scale=(1 << 21) + 8188)]),
    ("eat_block_mm", MM, [
        dict(y=A[0] + 12), dict(y=A[1] + 4), dict(y=A[2] + 8), dict(xs=(1 << 22) + 508), dict(ws=(1 << 22) + 508),
        dict(offsets=(1 << 22) + 508), dict(y=(1 << 20) + 254), dict(transposed=1, y=A[0] + 12)]),
    ("eat_block_mm_grad", MGRAD, [
        dict(dw=A[0] + 508), dict(dw=A[1] + 508), dict(dw=A[2] + 8), dict(gs=(1 << 22) + 16380),
        dict(xs=(1 << 22) + 16380), dict(offsets=(1 << 22) + 16380)]),
    ("eat_swiglu", GLU, [
        dict(h_dtype=FP8, scale=A[0] + 1020), dict(h_dtype=FP8, scale=A[1] + 252), dict(h=A[0] + 1022)]),
    ("eat_swiglu_grad", GLUGRAD, [dict(dgu=A[0] + 1022), dict(dgu=A[1] + 510)]),
]


@pytest.mark.parametrize("fn,base,kw", [(f, b, k) for f, b, cs in OVERLAPS for k in cs])
def test_an_output_that_overlaps_another_array(lib, fn, base, kw):
    _refused(lib, fn, {**base, **kw}.values(), "overlaps")
