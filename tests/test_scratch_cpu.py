"""The build refuses every kernel that spills registers to scratch memory."""
import pytest

from paper_2609_22870_amd import _build

REMARKS = """x.hip:1:0: remark: Function Name: {name} [-Rpass-analysis=kernel-resource-usage]
x.hip:1:0: remark:     VGPRs: 128 [-Rpass-analysis=kernel-resource-usage]
x.hip:1:0: remark:     ScratchSize [bytes/lane]: {size} [-Rpass-analysis=kernel-resource-usage]
"""


@pytest.mark.parametrize("name", ["gemm_kernel", "rmsnorm_backward_kernel", "row_kernel"])
def test_any_kernel_that_spills_is_refused(name):
    _build.check_no_scratch("x.hip", REMARKS.format(name=name, size=0))
    with pytest.raises(RuntimeError, match=name):
        _build.check_no_scratch("x.hip", REMARKS.format(name="first", size=0) + REMARKS.format(name=name, size=264))
