"""The kernels of the operators without a context spill no registers: the products hold their tiles in them, and a spill inside the loop waits
for every load under way.  Checked on what the compiler reports, without a GPU."""
import os
import shutil

import pytest

from tests.test_registers_host import HIPCC, test_no_spills as no_spills


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs the HIP compiler")
@pytest.mark.parametrize("source,kernels", [
    ("mx_gemm.hip", ("mx_gemm_tiles", "mx_gemm_split")),
    ("mx_quant.hip", ("mx_round_rows", "mx_round_tiles")),
    ("route.hip", ("route_rows", "route_finish", "route_back_rows")),
])
def test_operators_do_not_spill(source, kernels):
    no_spills(source, kernels)
