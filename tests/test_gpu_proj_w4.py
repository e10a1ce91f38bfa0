"""The product with 4-bit weights against its definition in 64 bits: groups of every size, row counts around the 16 rows of an operand,
reductions that end inside a unit of 128, one to many outputs, both types of x and of y."""
import pytest
import torch

import paper_2604_23108_amd as M
from gpu_harness import GuardBands

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _case(T, n_in, n_out, group, zeros, x8, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(T * 7 + n_in + n_out + seed)
    codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = ((0.2 + torch.rand((n_out, n_in // group), generator=gen, device="cuda")) * 0.01).bfloat16()
    z = torch.randint(0, 16, scales.shape, generator=gen, device="cuda", dtype=torch.uint8) if zeros else None
    x = torch.randn((T, n_in), generator=gen, device="cuda")
    if x8:
        x_scale = x.abs().amax(1) / 448
        return (x / x_scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8), x_scale, codes, scales, z
    return x.bfloat16(), None, codes, scales, z


def _want(x, x_scale, codes, scales, z, group):
    n_out = codes.shape[0]
    xd = x.double() if x_scale is None else x.view(torch.float8_e4m3fn).double() * x_scale.double()[:, None]
    c = torch.stack([codes & 15, codes >> 4], 2).reshape(n_out, -1, group).double()
    zd = 8.0 if z is None else z.double()[:, :, None]
    s = scales.double()[:, :, None]
    y = xd @ ((c - zd) * s).reshape(n_out, -1).T.contiguous()
    # what the sums add: (16 + c) x and (16 + z) x of a group, four products in a chain, then the groups, then four waves
    size = xd.abs() @ ((32 + c + zd) * s).reshape(n_out, -1).T.contiguous()
    return y, (12 + c.shape[1]) * U * size


def _check(got, y, off, y_dtype):
    bound = off + (2.0 ** -8 * y.abs() if y_dtype == M.BF16 else 0)
    assert got.isfinite().all() and ((got.double() - y).abs() <= bound).all(), float(((got.double() - y).abs() - bound).max())


def _run(T, n_in, n_out, group, zeros, x8, y_dtype):
    x, x_scale, codes, scales, z = _case(T, n_in, n_out, group, zeros, x8)
    cfg, g = M.ProjConfig(T, n_in, n_out, group=group, x_dtype=M.E4M3 if x8 else M.BF16, y_dtype=y_dtype), GuardBands()
    y = g.wrap(torch.empty((T, n_out), dtype=torch.float32 if y_dtype == M.F32 else torch.bfloat16, device="cuda"), "y").fill_(float("nan"))
    print(f"[proj] T={T} {n_in}->{n_out} group={group} zeros={zeros} x8={x8}", flush=True)
    M.mohge_proj_w4(cfg, x, x_scale, codes, scales, z, y)
    _check(y, *_want(x, x_scale, codes, scales, z, group), y_dtype)
    g.check()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros,x8,y_dtype", [(False, False, M.BF16), (True, False, M.F32), (True, True, M.F32), (False, True, M.BF16)])
@pytest.mark.parametrize("T", [1, 2, 5, 15, 16, 17, 32])
def test_rows_groups_and_types(T, group, zeros, x8, y_dtype):
    for n_in, n_out in ((group, 1), (3 * group, 17), (1408, 200)):
        _run(T, n_in, n_out, group, zeros, x8, y_dtype)


# reductions of 1, 3, 5 groups of 32 (a unit of 128 cut short), around the staged rows, long; outputs around 16, 64 and where waves no
# longer share rows
@pytest.mark.parametrize("T,n_in,n_out,group", [(1, 32, 16, 32), (3, 96, 15, 32), (32, 160, 64, 32), (1, 1344, 65, 64), (32, 992, 63, 32),
                                                (32, 1024, 33, 128), (31, 1152, 128, 128), (9, 3648, 100, 64), (1, 32896, 40, 128),
                                                (32, 33280, 16, 64), (4, 64, 32768, 64), (32, 96, 32769, 32), (1, 128, 70001, 128),
                                                (17, 320, 40007, 64), (2, 4096, 6145, 128)])
def test_sizes(T, n_in, n_out, group):
    _run(T, n_in, n_out, group, True, False, M.F32)


def test_weights_past_32_bit_offsets():
    """More than 2^31 bytes of codes: the last rows against the definition."""
    T, n_in, group = 3, 8192, 128
    n_out = 2 ** 31 // (n_in // 2) + 40
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = ((0.2 + torch.rand((n_out, n_in // group), generator=gen, device="cuda")) * 0.01).bfloat16()
    x = torch.randn((T, n_in), generator=gen, device="cuda").bfloat16()
    y = torch.empty((T, n_out), device="cuda")
    print("[proj] large", flush=True)
    M.mohge_proj_w4(M.ProjConfig(T, n_in, n_out, y_dtype=M.F32), x, None, codes, scales, None, y)
    for part in (slice(0, 64), slice(n_out - 64, n_out)):
        _check(y[:, part], *_want(x, None, codes[part], scales[part], None, group), M.F32)


def test_weights_quantised_by_the_package():
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn((300, 640), generator=gen, device="cuda") * 0.02
    x = torch.randn((6, 640), generator=gen, device="cuda").bfloat16()
    for group, zeros in ((128, False), (32, True)):
        codes, scales, z = M.quantize_w4(w, group, zeros)
        p = M.ProjW4(M.ProjConfig(6, 640, 300, group=group), codes, scales, z)
        y = p.forward(x)
        _check(y, *_want(x, None, codes, scales, z, group), M.BF16)
        # and near the product with the weights that were quantised: a step is at most max / 7, uniform errors of half a step
        full = x.double() @ w.double().T.contiguous()
        assert (y.double() - full).norm() <= 0.25 * full.norm()


def test_no_rows_and_rows_of_extremes():
    cfg = M.ProjConfig(0, 256, 48, group=64)
    x, _, codes, scales, z = _case(0, 256, 48, 64, True, False)
    M.mohge_proj_w4(cfg, x, None, codes, scales, z, torch.empty((0, 48), dtype=torch.bfloat16, device="cuda"))
    # infinities and NaN of one row of x stay in that row
    x, _, codes, scales, z = _case(4, 256, 48, 64, True, False)
    y = torch.empty((4, 48), dtype=torch.bfloat16, device="cuda")
    cfg = M.ProjConfig(4, 256, 48, group=64)
    M.mohge_proj_w4(cfg, x, None, codes, scales, z, y)
    bad = x.clone()
    bad[1, 5], bad[2, 200] = float("nan"), float("inf")
    y2 = torch.empty_like(y)
    M.mohge_proj_w4(cfg, bad, None, codes, scales, z, y2)
    assert torch.equal(y2[[0, 3]], y[[0, 3]]) and not y2[1:3].isfinite().any()


def test_same_bits_every_time_on_any_stream_and_in_a_graph():
    x, _, codes, scales, z = _case(7, 2560, 1000, 64, True, False)
    p = M.ProjW4(M.ProjConfig(7, 2560, 1000, group=64), codes, scales, z)
    want = p.forward(x).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.forward(x)
    torch.cuda.synchronize()
    assert torch.equal(p.y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(x)
    for i in range(3):
        x.mul_(1.5)
        eager = p.forward(x).clone()
        p.y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.y, eager), i
