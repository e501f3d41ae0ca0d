"""Host checks of a Muon step's factors, which the kernels take in 32 bits."""
import ctypes

import pytest

import __graft_entry__ as G
import paper_2609_34325_gb300 as P


@pytest.fixture(scope="module")
def lib():
    G.build()
    return P.load_library()


@pytest.mark.parametrize("lr,decay", [(1e39, 0.0), (-1e39, 0.0), (1e300, 0.0), (1e30, 1e30),
                                      (1e-300, float("inf")), (0.0, float("inf")),
                                      (0.0, float("nan")), (1e200, 1e200)])
def test_factors_past_32_bits_are_refused(lib, lr, decay):
    l = P._MatrixListC(data=256, chunks=1, x_tiles=2, symmetric=1, outputs=1, tiles=10,
                       diagonals=1, count=1, has_params=1, has_outs=1, large=1, parts=1)
    assert lib.dora_muon_step(ctypes.byref(l), lr, 0.9, 1, decay, 5, None, None, None) == 1
