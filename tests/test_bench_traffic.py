"""The bench's captured DRAM traffic belongs to the sources that are built."""
import os

import pytest

import bench as B

CSRC = os.path.join(B.ROOT, "paper_2609_34325_gb300", "csrc")


@pytest.mark.parametrize("source,captured", [("gemm_tcgen05.cu", B.NCU_GEMM_BYTES_PER_ROW),
                                             ("token_ops.cu", B.NCU_TRAFFIC_SELECT_COMPACT)])
def test_the_captured_traffic_is_that_of_the_present_sources(source, captured):
    # a change of these kernels, or of a header of theirs, wants a new capture: without it
    # the bench reports no traffic
    assert B.sha256_of(os.path.join(CSRC, source)) in captured
