"""8-bit rows bit by bit: scale = max|x| * (1/448) and code = x * (1/scale), in fp32 rounded to nearest, on rows that hold every bf16
mantissa below every largest one, where exact ties between codes are common; for bf16 rows the codes are those of x / scale too."""
import pytest
import torch

import paper_2604_23108_amd as M

pytestmark = pytest.mark.gpu


def _rows():
    """Rows of 256 bf16 values: a largest one with each of the 128 mantissas, and 255 of all smaller mantissas over 12 binades."""
    mantissas = torch.arange(128, 256).float() / 128
    below = torch.cat([mantissas * 2.0 ** -k for k in range(12)])
    rows = []
    for top in mantissas:
        x = below[below <= top]
        x = torch.cat([x, x.new_zeros(-len(x) % 255)]).reshape(-1, 255)
        x[:, ::2] *= -1
        rows.append(torch.cat([top.expand(x.shape[0], 1), x], 1))
    return torch.cat(rows)


def _codes(x):
    top = x.abs().amax(-1)
    scale = torch.where(top > 0, (top * torch.tensor(1 / 448)).clamp(min=2.0 ** -126), torch.ones_like(top))
    return (x * (1 / scale)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), scale


@pytest.mark.parametrize("head", [64, 128, 256])
def test_append(head):
    x = _rows()
    x = torch.cat([x, x * 2.0 ** 100, x * 2.0 ** -100, x * 2.0 ** -126]).reshape(-1, 1, head)
    n, page = x.shape[0], 64
    pages = -(-n // page)
    cfg = M.CacheConfig(1, 1, 1, head, page, pages, pages, cache_dtype=M.E4M3)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    kp, vp = (torch.zeros((pages, 1, page, head), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((pages, 1, page), device="cuda") for _ in range(2))
    k, v = x.bfloat16().cuda(), (-x).bfloat16().cuda()
    one = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    M.mohge_cache_append(cfg, k, v, one(0, n), table, one(n), kp, vp, ks, vs)
    for rows, codes, scales in ((k, kp, ks), (v, vp, vs)):
        want, scale = _codes(rows.float().cpu()[:, 0])
        assert torch.equal(scales.reshape(-1)[:n].cpu(), scale)
        assert torch.equal(codes.reshape(-1, head)[:n].cpu(), want)
        assert torch.equal(want, (rows.float().cpu()[:, 0] / scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("dtype", [M.BF16, M.F32])
def test_norm(dtype):
    x = _rows()
    T, d = x.shape
    t = torch.bfloat16 if dtype == M.BF16 else torch.float32
    gen = torch.Generator().manual_seed(1)
    w = torch.randn(d, generator=gen) if dtype == M.F32 else torch.ones(d)
    cfg = M.NormConfig(T, d, dtype=dtype, y_dtype=M.E4M3)
    codes, scale, rstd = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    M.mohge_rmsnorm(cfg, x.to(t).cuda(), None, w.cuda(), None, codes, scale, rstd)
    want, want_scale = _codes(x * w * rstd.cpu()[:, None])
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(codes.cpu(), want)
