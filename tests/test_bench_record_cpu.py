"""bench.py reports the HBM bytes of the GEMM from a committed counter record, and
nothing where the GEMM's sources changed since it was taken: the record is that of these
sources (else its profile says how to take it again)."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_the_record_is_of_these_sources():
    import bench

    traffic = bench.recorded_traffic("8b_ffn_up_fwd_blockwise")
    # 16384 x 4096 x 12288: every operand and the output at least once
    assert traffic is not None and traffic > 16384 * 4096 + 12288 * 4096 + 2 * 16384 * 12288
