"""Long rows of the attention, where stretches and their joins could lose or double a tile: planted values in which every 16 positions show, one
position that takes all the weight at every kind of boundary, and random ones against a bound that counts what one wave really adds up."""
import math

import pytest
import torch

import paper_2604_23108_amd as M
from test_gpu_cache import KINDS, TYPES, U, _filled, _values

pytestmark = pytest.mark.gpu

# (lengths, kv heads, query heads of each, head size, page)
LONG = [([70000, 70000], 1, 4, 128, 128), ([131072], 1, 1, 128, 64), ([40001, 7, 0], 2, 8, 64, 16), ([20011, 9000], 2, 3, 256, 32), ([16000], 8, 4, 128, 64),
        ([1531], 4, 4, 64, 16), ([3000 + 977 * i for i in range(29)], 2, 16, 64, 16)]


def _config(lens, kv, group, head, page, dtype, cache):
    pages = sum(-(-n // page) for n in lens) + 1
    return M.CacheConfig(len(lens), group * kv, kv, head, page, pages, -(-max(lens) // page), dtype=dtype, cache_dtype=cache)


def _attend(cfg, q, table, lens, kp, vp, ks, vs, scale):
    out = torch.full((cfg.n_seqs, cfg.n_heads, cfg.head_size), float("nan"), dtype=TYPES[cfg.dtype], device="cuda")
    lse = torch.full(out.shape[:2], float("nan"), device="cuda")
    ws = torch.zeros(M.mohge_cache_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, ks, vs, scale, out, lse, ws)
    return out, lse


def _put(cfg, table, b, positions, rows, pages, scales):
    """rows [positions, head] into every kv head of the sequence's positions (numbers that E4M3 holds, with a scale of 1)."""
    page, slot = table[b].long()[positions // cfg.page_size], positions % cfg.page_size
    rows = rows[:, None].expand(-1, cfg.n_kv_heads, -1)
    if scales is not None:
        rows = rows.to(torch.float8_e4m3fn).view(torch.uint8)
        scales[page, :, slot] = 1.0
    pages[page, :, slot] = rows.to(pages.dtype)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,kv,group,head,page", LONG)
def test_every_16_positions_count_once(lens, kv, group, head, page, dtype, cache):
    """Scores of 0, and a 1 in element (position / 16) % head of every value: all sums are whole numbers below 2^24, exact, and every element
    is its number of positions over the length: two roundings and that of the output.  An element has at most 65 tiles of 16."""
    cfg = _config(lens, kv, group, head, page, dtype, cache)
    q, table, n, kp, vp, ks, vs = _filled(cfg, lens)
    for b, length in enumerate(lens):
        at = torch.arange(length, device="cuda")
        if length:
            _put(cfg, table, b, at, torch.nn.functional.one_hot(at // 16 % head, head).float(), vp, vs)
    print(f"[attention] tiles {lens[:3]} head={head} {cache}", flush=True)
    out, lse = _attend(cfg, torch.zeros_like(q), table, n, kp, vp, ks, vs, 1.0)
    for b, length in enumerate(lens):
        if length == 0:
            continue
        want = torch.bincount(torch.arange(length, device="cuda") // 16 % head, minlength=head).double() / length
        err = (out[b].double() - want).abs()
        assert (err <= (4 * U + (2.0 ** -8 if dtype == M.BF16 else 0)) * want).all(), (b, float((err / want.clamp(min=1e-9)).max()))
        assert ((lse[b].double() - math.log(length)).abs() <= 8 * U * (1 + math.log(length))).all()


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,kv,group,head,page", LONG)
def test_one_position_takes_all(lens, kv, group, head, page, dtype, cache):
    """A key whose score is past all others by more than 2^7: the output is its value, bit by bit."""
    cfg = _config(lens, kv, group, head, page, dtype, cache)
    q, table, n, kp, vp, ks, vs = _filled(cfg, lens)
    one, b = torch.ones(1, head, device="cuda"), max(range(len(lens)), key=lambda i: lens[i])
    if ks is not None:
        ks.nan_to_num_(1.0).clamp_(max=1.5)
    q = torch.full_like(q, 4.0)
    length = lens[b]
    marks = [0, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 383, 384, length // 3, length // 2, length - 129, length - 65, length - 33, length - 17, length - 1]
    step = max(1, length // 37) | 1
    marks = sorted({p for p in marks + list(range(0, length, step)) if 0 <= p < length})
    print(f"[attention] {len(marks)} positions of {lens[:3]} head={head} {cache}", flush=True)
    for p in marks:
        at = torch.tensor([p], device="cuda")
        page_of, slot = int(table[b, p // page]), p % page
        kept = kp[page_of, :, slot].clone(), None if ks is None else ks[page_of, :, slot].clone()
        _put(cfg, table, b, at, one * 16, kp, ks)
        out, lse = _attend(cfg, q, table, n, kp, vp, ks, vs, head ** -0.5)
        value = _values(vp[page_of, :, slot], None if vs is None else vs[page_of, :, slot])          # [kv heads, head]
        want = value.repeat_interleave(group, 0)
        err = (out[b].double() - want).abs()
        # E4M3: value and scale are a product, whose two bf16 parts keep 2^-17 of it; other types exactly
        assert (err <= (0 if cache != M.E4M3 else 2.0 ** -8 + 2.0 ** -16) * want.abs()).all(), p
        assert ((lse[b].double() - 64 * head ** 0.5).abs() <= 4 * U * 64 * head ** 0.5).all(), p
        kp[page_of, :, slot] = kept[0]
        if ks is not None:
            ks[page_of, :, slot] = kept[1]


def _chain(cfg, lens):
    """Roundings in a row, in units of U: what a wave adds up (its tiles of a stretch of all units, by half as much more where a row is kept
    whole; per tile two products of at most 8 steps, each cut off at 2 U, and a rescaling), its fourth of the parts (three each), waves and lanes."""
    halves = {M.F32: 2 if cfg.head_size == 64 else 1, M.BF16: 2, M.E4M3: 1 if cfg.head_size == 256 else 2}[cfg.cache_dtype]
    unit = 64 * halves
    rows = cfg.n_kv_heads * -(-(cfg.n_heads // cfg.n_kv_heads) // 16)
    units = [max(1, -(-n // unit)) for n in lens]
    per = max(-(-sum(units) * rows // 256), 2)                # (256 workgroups at least)
    tiles = per + per // 2 + 2
    parts = -(-max(units) // per) + 2                         # (of a stretch of `per`; fewer where it is longer)
    parts = max(parts, -(-max(units) // max(1, -(-sum(units) * rows // 768))) + 2)
    return tiles * (2 * 8 * 2 + 1 + 8) + 3 * (parts / 4 + 1) + 24


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,kv,group,head,page", LONG)
def test_long_rows(lens, kv, group, head, page, dtype, cache):
    cfg = _config(lens, kv, group, head, page, dtype, cache)
    q, table, n, kp, vp, ks, vs = _filled(cfg, lens, 3)
    scale, D, S = head ** -0.5, head, page
    print(f"[attention] {lens[:3]} head={head} {cache}", flush=True)
    out, lse = _attend(cfg, q, table, n, kp, vp, ks, vs, scale)
    chain = _chain(cfg, lens) * U
    for b, length in enumerate(lens):
        if length == 0:
            continue
        pages = table[b, :-(-length // S)].long()
        rows = lambda x, s: _values(x[pages], None if s is None else s[pages]).transpose(0, 1).reshape(kv, -1, D)[:, :length]  # noqa: E731
        k, v, qd = rows(kp, ks), rows(vp, vs), q[b].double().reshape(kv, group, D)
        kt = k.transpose(1, 2).contiguous()
        z = scale * (qd @ kt)
        p = torch.softmax(z, 2)
        want, want_lse = p @ v, torch.logsumexp(z, 2)
        # a score's error is its own, of its products' sizes: D / 4 of them in a chain, the scale, the maximum, the exponential
        score = ((D / 4 + 12) * scale * (qd.abs() @ kt.abs()) + 4) * U
        mean = (p * score).sum(2)                             # ... and that of the sum of weights
        split = 2.0 ** -16 if dtype == M.BF16 else 0.0        # what the two parts of a weight leave
        bound = (p * score) @ v.abs() + (mean + 2 * chain + split)[:, :, None] * (p @ v.abs()) + (2.0 ** -8 * want.abs() if dtype == M.BF16 else 0)
        err = (out[b].double().reshape(kv, group, D) - want).abs()
        assert (err <= bound + 1e-37).all(), (b, float((err / bound).max()))
        err = (lse[b].double().reshape(kv, group) - want_lse).abs()
        assert (err <= mean + chain + 4 * U * want_lse.abs()).all(), (b, float(err.max()))
