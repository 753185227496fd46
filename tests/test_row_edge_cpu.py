"""The elements of a row of logits outside its whole 16-byte pieces, up to the longest
rows, under the sanitizers."""
import os

from test_sanitizers import CSRC, ROOT, SAN, build_and_run


def test_edges_of_rows(tmp_path):
    exe = str(tmp_path / "row_edge")
    build_and_run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__"] + SAN +
                  ["-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                   "-I", os.path.join(ROOT, "paper_2609_22870_amd", "csrc"),
                   os.path.join(CSRC, "row_edge_main.cpp"), "-o", exe], exe)
