"""The norm with the residual's addition against its definition in 64 bits: every row width that takes another number of threads
or pieces, both types, 8-bit rows, the gradient against the formula and against differences, aliased buffers, odd inputs."""
import pytest
import torch

import paper_2604_23108_amd as M
from gpu_harness import GuardBands

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                 # fp32 rounding
# A row's sum of squares: at most 8 terms per piece, four pieces, six steps of lanes and 16 waves in a chain, all positive; half of its
# relative error in rstd, a unit for the root, three products.
RSTD = (0.5 * (32 + 6 + 16) + 4) * U
HALF_BF16 = 2.0 ** -8          # half an ulp of a bf16 number, relative
EPS = 1e-6
TYPES = {M.BF16: torch.bfloat16, M.F32: torch.float32}

SHAPES = [(1, 8), (3, 64), (5, 504), (4, 512), (7, 520), (9, 1024), (2, 1032), (33, 1344), (1, 2048), (6, 2056), (130, 2560), (1, 4096),
          (3, 4104), (5, 8192), (2, 8200), (3, 16384), (2, 16392), (3, 32768), (1030, 512), (2051, 1024)]


def _inputs(T, d, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(T * 131 + d + seed)
    t = TYPES[dtype]
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return normal(T, d).to(t), (2 * normal(T, d)).to(t), 1 + 0.3 * normal(d), normal(T, d).to(t), normal(T, d).to(t)


def _forward(x, r, w):
    h = x.double() + (0 if r is None else r.double())
    rstd = 1 / torch.sqrt(h.square().mean(1) + EPS)
    return h, rstd, h * rstd[:, None] * w.double()


def _rounded(got, want, dtype, extra):
    bound = extra + (HALF_BF16 * want.abs() if dtype == M.BF16 else 0)
    assert got.isfinite().all() and ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() - bound).max())


@pytest.mark.parametrize("dtype", [M.BF16, M.F32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward_and_backward(T, d, dtype):
    x, r, w, dy, ds = _inputs(T, d, dtype)
    t = TYPES[dtype]
    cfg, g = M.NormConfig(T, d, dtype=dtype, eps=EPS), GuardBands()
    out = lambda name, shape, ty=t: g.wrap(torch.empty(shape, dtype=ty, device="cuda"), name)  # noqa: E731
    print(f"[norm] T={T} d={d} dtype={dtype}", flush=True)
    for res in (r, None):
        s, y, rstd = out("sum", (T, d)), out("y", (T, d)), out("rstd", (T,), torch.float32)
        M.mohge_rmsnorm(cfg, x, res, w, s, y, None, rstd)
        h, want_rstd, want = _forward(x, res, w)
        _rounded(s, h, dtype, U * h.abs())
        assert ((rstd.double() - want_rstd).abs() <= RSTD * want_rstd).all()
        _rounded(y, want, dtype, (RSTD + 3 * U) * want.abs() + 1e-37)
        # the backward pass reads what the forward pass stored
        for dsum in (ds, None):
            dx, dw = out("dx", (T, d)), out("dw", (d,), torch.float32)
            ws = out("ws", (M.mohge_norm_workspace_size(cfg),), torch.uint8)
            M.mohge_rmsnorm_bwd(cfg, dy, s, w, rstd, dsum, dx, dw, ws)
            n, gd = s.double() * rstd.double()[:, None], w.double() * dy.double()
            want_dx = rstd.double()[:, None] * (gd - n * (gd * n).mean(1, keepdim=True))
            # products and the sum of a row: at most 54 in a chain
            off = 64 * U * rstd.double()[:, None] * (gd.abs() + n.abs() * (gd * n).abs().mean(1, keepdim=True))
            if dsum is not None:
                want_dx = want_dx + dsum.double()
                off = off + 2 * U * want_dx.abs()
            _rounded(dx, want_dx, dtype, off)
            terms = dy.double() * n
            # the rows of a workgroup in a chain, then the workgroups' sums
            bound = (T / 512 + 1 + 32 + 16 + 3) * U * terms.abs().sum(0)
            assert ((dw.double() - terms.sum(0)).abs() <= bound).all()
    torch.cuda.synchronize()
    g.check()


@pytest.mark.parametrize("dtype", [M.BF16, M.F32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_rows_of_8_bit_codes(T, d, dtype):
    x, r, w, _, _ = _inputs(T, d, dtype, 1)
    if T > 2:
        x[1], r[1] = 0, 0                                  # a row of zeros
        x[2] *= 1e-3
        r[2] *= 1e-3
    cfg, g = M.NormConfig(T, d, dtype=dtype, y_dtype=M.E4M3, eps=EPS), GuardBands()
    codes, scale = g.wrap(torch.empty((T, d), dtype=torch.uint8, device="cuda"), "codes"), g.wrap(torch.empty(T, device="cuda"), "scale")
    s = torch.empty_like(x)
    print(f"[norm 8 bit] T={T} d={d} dtype={dtype}", flush=True)
    M.mohge_rmsnorm(cfg, x, r, w, s, codes, scale)
    h, _, want = _forward(x, r, w)
    _rounded(s, h, dtype, U * h.abs())
    top = want.abs().amax(1)
    want_scale = torch.where(top > 0, top / 448, torch.ones_like(top))
    assert ((scale.double() - want_scale).abs() <= (RSTD + 4 * U) * want_scale).all()
    got = codes.view(torch.float8_e4m3fn).double() * scale.double()[:, None]
    # half of the distance between codes: 2^-4 of the value, 2^-10 of the scale below the normal ones
    bound = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * want_scale[:, None]) + (2 * RSTD + 8 * U) * want.abs()
    assert got.isfinite().all() and ((got - want).abs() <= bound).all()
    g.check()


def test_buffers_may_be_the_inputs():
    x, r, w, dy, ds = _inputs(37, 1344, M.BF16, 2)
    cfg = M.NormConfig(37, 1344)
    s, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(37, device="cuda")
    M.mohge_rmsnorm(cfg, x, r, w, s, y, None, rstd)
    for into in (0, 1):
        a, b, y2 = x.clone(), r.clone(), torch.empty_like(x)
        M.mohge_rmsnorm(cfg, a, b, w, (a, b)[into], y2)
        assert torch.equal((a, b)[into], s) and torch.equal(y2, y)
    dx, dw = torch.empty_like(x), torch.empty(1344, device="cuda")
    ws = torch.empty(M.mohge_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    M.mohge_rmsnorm_bwd(cfg, dy, s, w, rstd, ds, dx, dw, ws)
    for into in (0, 1):
        a, b, dw2 = dy.clone(), ds.clone(), torch.empty_like(dw)
        M.mohge_rmsnorm_bwd(cfg, a, s, w, rstd, b, (a, b)[into], dw2, ws)
        assert torch.equal((a, b)[into], dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("T,d", [(5, 264), (64, 1024)])
def test_gradient_against_differences(T, d):
    """The directional derivative of sum(dy * y) + sum(ds * sum) by central differences of the forward pass in fp32."""
    x, r, w, dy, ds = _inputs(T, d, M.F32, 3)
    gen = torch.Generator(device="cuda").manual_seed(5)
    ux, uw = torch.randn(x.shape, generator=gen, device="cuda"), torch.randn(w.shape, generator=gen, device="cuda")
    norm = M.ResidualNorm(M.NormConfig(T, d, dtype=M.F32, eps=EPS), w, backward=True)

    def loss(step_x, step_w):
        n = M.ResidualNorm(M.NormConfig(T, d, dtype=M.F32, eps=EPS), w + step_w * uw)
        y = n.forward(x + step_x * ux, r)
        return float((dy.double() * y.double()).sum() + (ds.double() * n.sum.double()).sum())

    norm.forward(x, r)
    dx, dw = norm.backward(dy, ds).double(), norm.dweight.double()
    eps = 1e-2
    # the derivative of such a sum is of the order sqrt(T d); its third one times eps^2 / 6 and the rounding of the two
    # losses, U sqrt(T d) / eps each, stay below these shares of it
    by_x, by_w = (loss(eps, 0) - loss(-eps, 0)) / (2 * eps), (loss(0, eps) - loss(0, -eps)) / (2 * eps)
    assert abs(by_x - float((dx * ux).sum())) <= 3e-4 * (T * d) ** 0.5
    assert abs(by_w - float((dw * uw).sum())) <= 3e-4 * (T * d) ** 0.5


def test_rows_of_zeros_infinities_and_nothing():
    d = 1024
    x = torch.randn(5, d, device="cuda").bfloat16()
    x[0] = 0
    x[1, 7] = float("inf")
    x[2, 9] = float("nan")
    w = torch.ones(d, device="cuda")
    for eps in (EPS, 0.0):
        y, rstd = torch.empty_like(x), torch.empty(5, device="cuda")
        M.mohge_rmsnorm(M.NormConfig(5, d, eps=eps), x, None, w, None, y, None, rstd)
        want = (x.float() * (x.float().square().mean(1) + eps).rsqrt()[:, None])
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y[0].float().nan_to_num(9.0), want[0].nan_to_num(9.0))
        assert y[3:].isfinite().all() and rstd[1] == 0
        codes, scale = torch.empty((5, d), dtype=torch.uint8, device="cuda"), torch.empty(5, device="cuda")
        M.mohge_rmsnorm(M.NormConfig(5, d, y_dtype=M.E4M3, eps=eps), x, None, w, None, codes, scale)
        back = codes.view(torch.float8_e4m3fn).float() * scale[:, None]
        assert not back[1].isfinite().all() and not back[2].isfinite().all() and back[3:].isfinite().all()
    # no rows: nothing is written but the sum over them
    dw = torch.full((d,), 7.0, device="cuda")
    cfg = M.NormConfig(0, d)
    e, f = torch.empty((0, d), dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    M.mohge_rmsnorm(cfg, e, None, w, None, e)
    M.mohge_rmsnorm_bwd(cfg, e, e, w, f, None, e, dw, torch.empty(M.mohge_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda"))
    assert (dw == 0).all()


def test_same_bits_every_time_on_any_stream_and_in_a_graph():
    T, d = 1111, 1344
    x, r, w, dy, ds = _inputs(T, d, M.BF16, 4)
    norm = M.ResidualNorm(M.NormConfig(T, d), w, backward=True)

    def step():
        norm.forward(x, r)
        norm.backward(dy, ds)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (norm.sum, norm.y, norm.rstd, norm.dx, norm.dweight)]

    step()
    want = results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.add_(0.25)
        step()
        eager = results()
        for t in (norm.sum, norm.y, norm.rstd, norm.dx, norm.dweight):
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), eager)), i
