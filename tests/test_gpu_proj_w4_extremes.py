"""The product with 4-bit weights where x holds infinities, NaN and numbers near the largest: what the definition gives, in every form of the
kernel."""
import pytest
import torch

import paper_2604_23108_amd as M
from test_gpu_proj_w4 import _case, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,zeros", [(128, False), (64, True), (32, False)])
@pytest.mark.parametrize("T,n_in,n_out", [(4, 640, 48), (4, 4224, 100), (8, 640, 48), (16, 4224, 100), (16, 640, 48), (32, 640, 48), (32, 4224, 100),
                                          (16, 640, 20481), (32, 640, 20481), (16, 640, 49153), (32, 640, 49153)])
def test_infinities_and_large_numbers(T, n_in, n_out, group, zeros):
    x, _, codes, scales, z = _case(T, n_in, n_out, group, zeros, False, 5)
    inf = float("inf")
    x[0, 3] = inf
    x[1, 130], x[1, 600] = -inf, inf
    x[2, 7] = float("nan")
    x[3, 500] = 2e37                                     # times 15 it is finite, times 31 it is not
    x[T - 1, n_in - 1] = -inf if T > 4 else x[T - 1, n_in - 1]
    want, off = _want(x, None, codes, scales, z, group)
    print(f"[proj] extremes T={T} {n_in}->{n_out} group={group}", flush=True)
    for dtype in (M.F32, M.BF16):
        y = torch.empty((T, n_out), dtype=torch.float32 if dtype == M.F32 else torch.bfloat16, device="cuda")
        M.mohge_proj_w4(M.ProjConfig(T, n_in, n_out, group=group, y_dtype=dtype), x, None, codes, scales, z, y)
        y = y.double()
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.isinf(), want.isinf())
        assert torch.equal(y[y.isinf()], want[want.isinf()]) and y[0].isinf().any() and y[2].isnan().all()
        assert y[3].isfinite().all() and y[3].abs().max() > 1e35
        there = want.isfinite()
        bound = off + (2.0 ** -8 * want.abs() if dtype == M.BF16 else 0)
        assert ((y - want).abs()[there] <= bound[there]).all()
    if T > 4:
        others = [*range(4, T - 1)]
        assert y[others].isfinite().all() and not y[T - 1].isfinite().any()


def test_codes_of_nan():
    x, x_scale, codes, scales, z = _case(5, 1344, 70, 64, True, True)
    x[1, 77], x[4, 0] = 127, 255
    y = torch.empty((5, 70), device="cuda")
    M.mohge_proj_w4(M.ProjConfig(5, 1344, 70, group=64, x_dtype=M.E4M3, y_dtype=M.F32), x, x_scale, codes, scales, z, y)
    assert y[[1, 4]].isnan().all() and y[[0, 2, 3]].isfinite().all()
