"""Every kernel that is compiled for the GPU has a launch: a variant that no size
chooses is device code without the host stub that a launch brings."""
import os
import re
import subprocess

import pytest

from paper_2609_22870_amd import _build


@pytest.mark.parametrize("src", ["loss.hip", "norm.hip", "requantize.hip"])
def test_every_kernel_is_launched(src, tmp_path):
    obj = str(tmp_path / "out.o")
    r = subprocess.run([_build.HIPCC] + _build.FLAGS + _build.EXTRA.get(src, []) +
                       ["-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(_build.CSRC, src), "-o", obj],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = set(re.findall(r"Function Name: (\S+)", r.stderr))
    symbols = {line.split()[-1] for line in
               subprocess.run(["nm", obj], capture_output=True, text=True, check=True).stdout.splitlines()}
    assert kernels and not kernels - symbols, sorted(kernels - symbols)
