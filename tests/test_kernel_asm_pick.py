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
