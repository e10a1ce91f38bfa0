"""The norm where workgroups walk several rows each (three turns and more, the last one ragged), against the same definition and bounds: every
number of threads and pieces, one and two workgroups per compute unit, more parts of the weight's gradient than one pass adds."""
import pytest

import paper_2604_23108_amd as M
import test_gpu_norm as N

pytestmark = pytest.mark.gpu


# threads per row x pieces: 64x1, 64x2 (388 workgroups), 128x2, 128x2 with 512 workgroups, 512x1, 1024x1, 1024x2 and 1024x4 (no row ahead)
@pytest.mark.parametrize("dtype", [M.BF16, M.F32])
@pytest.mark.parametrize("T,d", [(3701, 512), (6203, 1024), (1501, 2048), (8191, 2048), (601, 2560), (601, 4096), (601, 8192), (601, 8200),
                                 (601, 16384), (601, 16392), (601, 32768), (777, 2048), (8191, 1344)])
def test_several_rows_per_workgroup(T, d, dtype):
    N.test_forward_and_backward(T, d, dtype)


@pytest.mark.parametrize("T,d", [(3701, 504), (1501, 2056)])
def test_8_bit_rows(T, d):
    N.test_rows_of_8_bit_codes(T, d, M.BF16)
