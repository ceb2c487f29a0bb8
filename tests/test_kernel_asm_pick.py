"""Only kernels that are asked for given ids' logits hold the code that picks them out (whole 16-byte stores of a
tile's columns into LDS, which nothing else in a logits kernel makes)."""
import os

import pytest

from tests.test_kernel_asm import CSRC, _body, _compile

PICK = "_ZN6fastrl14lm_pick_kernelENS_10GemmParamsE"
REDO = "_ZN6fastrl14lm_redo_kernelENS_10GemmParamsE"
GEMM = "_ZN6fastrl14lm_gemm_kernelItLi0EEEvNS_10GemmParamsE"


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    return _compile(os.path.join(CSRC, "lmhead.hip"), tmp_path_factory.mktemp("asm"))


@pytest.mark.parametrize("kernel, picks", [(PICK, True), (REDO, False), (GEMM, False)])
def test_pick_code_where_it_runs(asm, kernel, picks):
    assert any(op == "ds_write_b128" for _, op, _ in _body(asm, kernel)) == picks


@pytest.mark.parametrize("width, waves", [(32, 1), (64, 2)])
def test_float32_pick_code_where_it_runs(asm, width, waves):
    name = "_ZN6fastrl15f32_gemm_kernelILi0ELi256ELi%dELi4ELi%dELi2ELb%dEEEvNS_10GemmParamsE"
    for picks in (False, True):
        ops = [op for _, op, _ in _body(asm, name % (width, waves, picks))]
        assert any(op == "ds_write_b128" for op in ops) == picks
