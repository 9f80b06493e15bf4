"""Results whose rows overlap are refused, without a GPU: several writers of one value have no result."""
import ctypes as C

import pytest

from paper_2312_17530_b200.build import build_library
from test_operators_recurrence_host import BACK, BACK_GOOD, ORTHO, ORTHO_GOOD, SCAN, SCAN_GOOD, call

from paper_2312_17530_b200 import binding


@pytest.fixture(scope="module")
def lib():
    build_library()
    return binding.lib()


# four sequences of ten steps, 64 channels; none of these strides is below the width
@pytest.mark.parametrize("seq,step", [(64, 64), (639, 64), (64, 255), (320, 64), (64 * 9, 64), (1000, 500), (1000, 1000), (100, 110), (1000, 330),
                                      (1 << 62, 1 << 62)])
def test_scan_refuses_results_that_overlap(lib, seq, step):
    assert call(lib.rsdgc_gated_scan_forward, SCAN, SCAN_GOOD, ys=seq, yt=step) == -1
    assert call(lib.rsdgc_gated_scan_backward, BACK, BACK_GOOD, dxs=seq, dxt=step) == -1
    assert call(lib.rsdgc_gated_scan_backward, BACK, BACK_GOOD, dgs=seq, dgt=step) == -1


@pytest.mark.parametrize("matrix,row", [(40, 40), (1199, 40), (40, 79), (400, 40), (500, 50), (100, 130)])
def test_orthogonalize_refuses_results_that_overlap(lib, matrix, row):
    """Two matrices of 30 x 40"""
    assert call(lib.rsdgc_orthogonalize, ORTHO, ORTHO_GOOD, outm=matrix, outr=row) == -1
