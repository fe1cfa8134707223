"""The kernels of plain bf16 experts spill no registers.  Checked on what the compiler reports, without a GPU."""
import shutil

import pytest

from tests.test_registers_host import HIPCC, test_no_spills as no_spills


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs the HIP compiler")
@pytest.mark.parametrize("source,kernels", [
    ("expert_gemm.hip", ("expert_gemm_tiles", "expert_gemm_few", "expert_weights_add")),
    ("expert_rows.hip", ("expert_sort_count", "expert_sort_place", "expert_rows_out", "expert_rows_sum", "expert_rows_back")),
])
def test_experts_do_not_spill(source, kernels):
    no_spills(source, kernels)
