"""Block-scaled products and sorted rows: calls that the C entry points refuse, host only."""
import pytest

from paper_2609_33614_gb300 import build, eat
from test_experts_host import A, MGRAD, MM

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
