"""The kernels over histories and of drawing keep their registers (see test_host_operator_registers.py)."""
import pytest

from test_host_operator_registers import test_no_kernel_spills as no_kernel_spills


@pytest.mark.parametrize("file,at_least", [("op_rotary.hip", 20), ("op_sample.hip", 8), ("op_attention.hip", 8), ("op_attention_bwd.hip", 20), ("op_cache.hip", 30)])
def test_no_kernel_over_histories_spills(tmp_path, file, at_least):
    import shutil
    from test_host_operator_registers import HIPCC
    if shutil.which(HIPCC) is None:
        pytest.skip("no HIP compiler")
    no_kernel_spills(tmp_path, file, at_least)
