"""The wait states of the DMA loads (test_isa_hazards.py) in the products with something fused behind
them, whose kernels are compiled of their own (CPU)."""
import os

import pytest

from test_isa_hazards import _asm_for, _dma_problems, _functions, fbl_build


@pytest.mark.skipif(not os.path.exists(fbl_build.HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("src", ["head_gemm.hip", "linear_gemm_gelu.hip"])
def test_inline_dma_wait_states(src, tmp_path):
    checked, problems = _dma_problems(_functions(_asm_for(src, tmp_path)))
    assert checked > 0
    assert not problems, "\n".join(problems[:20])
