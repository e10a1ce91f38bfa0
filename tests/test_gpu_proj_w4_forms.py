"""Every form of the product with 4-bit weights over several batches and a last one that is cut short: shared staging with one and two blocks of weight
rows per wave, eight waves along the reduction; and rows of one sign, where the offset in front of the codes is largest against the result."""
import pytest
import torch

import paper_2604_23108_amd as M
from test_gpu_proj_w4 import U, _run, _want

pytestmark = pytest.mark.gpu


# 13 units of 128, or 13 and a half, or 13 and three quarters: three to thirteen batches and a shorter one
@pytest.mark.parametrize("group,n_in", [(128, 1664), (64, 1728), (32, 1760)])
@pytest.mark.parametrize("n_out", [20479, 20481, 49152, 49153, 65001])
@pytest.mark.parametrize("T", [5, 16, 17, 32])
def test_shared_staging(T, n_out, group, n_in):
    for zeros, x8, y_dtype in ((False, False, M.BF16), (True, True, M.F32), (False, True, M.F32), (True, False, M.BF16)):
        _run(T, n_in, n_out, group, zeros, x8, y_dtype)


# 33 and 65 units (and a part of one): uneven shares of the eight waves
@pytest.mark.parametrize("group,n_in", [(128, 4224), (64, 4288), (32, 8352), (128, 8320)])
@pytest.mark.parametrize("T", [1, 4, 5, 7, 8, 13, 16, 17, 32])
def test_eight_waves(T, group, n_in):
    for n_out in (33, 4096, 4097):
        for zeros, x8, y_dtype in ((False, False, M.F32), (True, True, M.BF16)):
            _run(T, n_in, n_out, group, zeros, x8, y_dtype)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("T,n_in,n_out", [(1, 4096, 300), (7, 4096, 300), (32, 1024, 300), (16, 1024, 20481), (32, 1024, 49153)])
@pytest.mark.parametrize("weights_too", [False, True])
def test_rows_of_one_sign(T, n_in, n_out, group, zeros, weights_too):
    """Were the matrix cores to cut sums off, all that they lose would have one sign.  A group's two sums, of (16 + c) x and of (16 + z) x, are added up in at most 16
    steps (8 products each) that cut off less than a unit (2 U) of what is there; a group's result then has three roundings, and the groups
    and waves one each."""
    gen = torch.Generator(device="cuda").manual_seed(T + n_in + n_out + group)
    codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = ((0.2 + torch.rand((n_out, n_in // group), generator=gen, device="cuda")) * 0.01).bfloat16()
    z = torch.randint(0, 9 if weights_too else 16, scales.shape, generator=gen, device="cuda", dtype=torch.uint8) if zeros else None
    if weights_too:
        codes |= 0x88                                    # 8 to 15
    x = torch.randn((T, n_in), generator=gen, device="cuda").abs().bfloat16()
    y = torch.empty((T, n_out), device="cuda")
    print(f"[proj] one sign T={T} {n_in}->{n_out} group={group} weights too: {weights_too}", flush=True)
    M.mohge_proj_w4(M.ProjConfig(T, n_in, n_out, group=group, y_dtype=M.F32), x, None, codes, scales, z, y)
    want, _ = _want(x, None, codes, scales, z, group)
    c = torch.stack([codes & 15, codes >> 4], 2).reshape(n_out, -1, group).double()
    zd = 8.0 if z is None else z.double()[:, :, None]
    s = scales.double()[:, :, None]
    size = lambda w: x.double() @ (w * s).reshape(n_out, -1).T.contiguous()  # noqa: E731
    with_offset, result = size(32 + c + zd), size((c - zd).abs())
    bound = 32 * U * with_offset + (n_in // group + 8 + 3) * U * result
    err = (y.double() - want).abs()
    print(f"  largest error / sum of |w x| {float((err / result).max()):.2e}, mean {float(((y.double() - want) / result).mean()):.2e}", flush=True)
    assert y.isfinite().all() and (err <= bound).all(), float((err / bound).max())
