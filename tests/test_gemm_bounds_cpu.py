"""What gemm_tile.h's MXFP4 tiles rest on is checked when they are compiled: the LDS reads of a step before its
first wait fit the counter that the wait reads."""
import os
import subprocess

import pytest

from paper_2609_22870_amd import _build

SOURCE = """
#include "gemm_tile.h"
namespace fp8q { namespace gemm_detail {
__global__ __launch_bounds__(256) void kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[TileLds<kPairMx4, %(bm)d, %(bn)d, %(wm)d, %(wn)d>::kBytes];
  gemm_tile<kPairMx4, %(bm)d, %(bn)d, %(wm)d, %(wn)d, false, 0>(g, lds, 0, 0);
}
} }
"""


@pytest.mark.parametrize("wn,fits", [(64, True), (128, False)])
def test_reads_in_flight(wn, fits, tmp_path):
    """A wave of 64 columns has 15 in flight, the counter's most; a wider one is refused."""
    src = tmp_path / "tile.hip"
    src.write_text(SOURCE % dict(bm=128, bn=2 * wn, wm=64, wn=wn))
    r = subprocess.run([_build.HIPCC] + _build.FLAGS + _build.EXTRA["gemm_mx4.hip"] +
                       ["--cuda-device-only", "-fsyntax-only", str(src)], capture_output=True, text=True)
    says = "reads of an MXFP4 step" in r.stderr
    assert says != fits and (r.returncode == 0 or not fits), r.stderr[-3000:]
