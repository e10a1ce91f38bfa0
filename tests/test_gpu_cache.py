"""The paged cache and the attention over it against their definitions in 64 bits: lengths from empty to several pieces, pages that end inside
a tile, groups of 1 to 32 query heads, all types, rows past a sequence's end full of NaN, page numbers out of range, offsets past
32 bits, lengths that change between replays of a graph."""
import math

import pytest
import torch

import paper_2604_23108_amd as M
from gpu_harness import GuardBands

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {M.BF16: torch.bfloat16, M.F32: torch.float32}


def _values(store, scale):
    return store.double() if scale is None else store.view(torch.float8_e4m3fn).double() * scale.double()[..., None]


def _filled(cfg, lens, seed=0, extra_pages=0):
    """Pages in a mixed order with random keys and values in the positions that the sequences have, NaN everywhere else; table
    entries that are not to be read hold numbers out of range."""
    gen = torch.Generator(device="cuda").manual_seed(seed + sum(lens) + cfg.head_size)
    S = cfg.page_size
    shape = (cfg.n_pages, cfg.n_kv_heads, S, cfg.head_size)
    order = torch.randperm(cfg.n_pages, generator=gen, device="cuda").tolist()
    table = torch.full((cfg.n_seqs, cfg.max_pages), 1 << 30, dtype=torch.int32)
    used = torch.zeros(cfg.n_pages, S, dtype=torch.bool)
    for b, n in enumerate(lens):
        for i in range(-(-n // S)):
            page = order.pop()
            table[b, i] = page
            used[page, :min(S, n - i * S)] = True
    used = used.cuda()[:, None, :, None]
    stores, scales = [], []
    for _ in range(2):
        x = torch.randn(shape, generator=gen, device="cuda")
        if cfg.cache_dtype == M.E4M3:
            stores.append(torch.where(used, x.to(torch.float8_e4m3fn).view(torch.uint8), torch.full_like(x, 127).byte()))
            s = 0.5 + torch.rand(shape[:3], generator=gen, device="cuda")
            scales.append(torch.where(used[..., 0], s, torch.full_like(s, float("nan"))))
        else:
            stores.append(torch.where(used, x, torch.full_like(x, float("nan"))).to(TYPES[cfg.cache_dtype]))
            scales.append(None)
    q = torch.randn((cfg.n_seqs, cfg.n_heads * cfg.head_size + 8), generator=gen, device="cuda").to(TYPES[cfg.dtype])
    q = q[:, :cfg.n_heads * cfg.head_size].view(cfg.n_seqs, cfg.n_heads, cfg.head_size)
    return q, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), stores[0], stores[1], scales[0], scales[1]


def _check(cfg, q, table, lens, kp, vp, ks, vs, scale, out, lse):
    G, Hk, D, S = cfg.n_heads // cfg.n_kv_heads, cfg.n_kv_heads, cfg.head_size, cfg.page_size
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        pages = table[b, :-(-n // S)].long()
        rows = lambda x, s: _values(x[pages], None if s is None else s[pages]).transpose(0, 1).reshape(Hk, -1, D)[:, :n]  # noqa: E731
        k, v = rows(kp, ks), rows(vp, vs)
        qd = q[b].double().reshape(Hk, G, D)
        kt = k.transpose(1, 2).contiguous()
        z = scale * (qd @ kt)
        p = torch.softmax(z, 2)
        want, want_lse = p @ v, torch.logsumexp(z, 2)
        # a score: its products four at a time in a chain, the scale and the maximum's subtraction, the exponential's unit; the
        # sums of weights and of products: positions of a wave in a chain, then waves and pieces
        size = abs(scale) * (qd.abs() @ kt.abs()).amax(2)
        score = (D / 4 + 12) * U * size + 4 * U
        chain = (n / 8 + 128) * U
        weight = 2 * score + chain + (2.0 ** -16 if cfg.dtype == M.BF16 else 0)        # bf16: what the two parts of a weight leave
        bound = (weight + chain)[:, :, None] * (p @ v.abs()) + (2.0 ** -8 * want.abs() if cfg.dtype == M.BF16 else 0)
        got = out[b].double().reshape(Hk, G, D)
        assert got.isfinite().all() and ((got - want).abs() <= bound + 1e-37).all(), (b, n, float(((got - want).abs() - bound).max()))
        err = (lse[b].double().reshape(Hk, G) - want_lse).abs()
        assert (err <= score + chain + 4 * U * want_lse.abs()).all(), (b, n, float(err.max()))


def _attend(cfg, lens, seed=0, scale=None):
    args = _filled(cfg, lens, seed)
    g = GuardBands()
    shape = (cfg.n_seqs, cfg.n_heads, cfg.head_size)
    out = g.wrap(torch.empty(shape, dtype=TYPES[cfg.dtype], device="cuda"), "out").fill_(float("nan"))
    lse = g.wrap(torch.empty(shape[:2], device="cuda"), "lse").fill_(float("nan"))
    ws = g.wrap(torch.empty(max(16, M.mohge_cache_workspace_size(cfg)), dtype=torch.uint8, device="cuda"), "workspace").zero_()
    scale = cfg.head_size ** -0.5 if scale is None else scale
    q, table, sl, kp, vp, ks, vs = args
    M.mohge_cache_attention(cfg, q, table, sl, kp, vp, ks, vs, scale, out, lse, ws)
    _check(cfg, *args, scale, out, lse)
    g.check()
    blocks = cfg.n_kv_heads * -(-(cfg.n_heads // cfg.n_kv_heads) // 16)
    assert (ws[:4 * cfg.n_seqs * blocks] == 0).all()              # the counters, for the next call
    return args, out, lse, ws


KINDS = [(M.BF16, M.BF16), (M.BF16, M.E4M3), (M.F32, M.F32)]
LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 127, 128, 129, 255, 300, 1000]


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("head", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_lengths_pages_and_types(dtype, cache, head, page):
    group, kv = {16: (4, 2), 32: (1, 3), 64: (7, 1), 128: (8, 2), 256: (16, 1)}[page]
    pages = sum(-(-n // page) for n in LENGTHS) + 2
    cfg = M.CacheConfig(len(LENGTHS), group * kv, kv, head, page, pages, 1024 // page, dtype=dtype, cache_dtype=cache)
    print(f"[attention] {dtype} {cache} head={head} page={page}", flush=True)
    _attend(cfg, LENGTHS)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("group,kv", [(2, 16), (15, 1), (16, 2), (17, 2), (32, 1), (128, 1)])
def test_query_heads(dtype, cache, group, kv):
    lens = [70, 0, 513]
    cfg = M.CacheConfig(3, group * kv, kv, 128, 16, 50, 40, dtype=dtype, cache_dtype=cache)
    print(f"[attention] {dtype} {cache} group={group}", flush=True)
    _attend(cfg, lens, 1)


# one sequence in many pieces, a few that share the grid unevenly, many short ones, a table far wider than the lengths, and more
# sequences than the machine has workgroups
@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,kv,page,columns", [([40001], 2, 64, 626), ([9000, 3, 0, 20011, 1], 4, 16, 1251), ([1] * 300, 2, 16, 1),
                                                  ([257], 8, 256, 4096), ([100 + i % 61 for i in range(700)], 3, 32, 8),
                                                  ([70000, 70000], 1, 128, 1000), ([0, 0, 0], 2, 16, 2)])
def test_long_and_many(dtype, cache, lens, kv, page, columns):
    pages = sum(-(-n // page) for n in lens) + 1
    cfg = M.CacheConfig(len(lens), 4 * kv, kv, 128, page, pages, columns, dtype=dtype, cache_dtype=cache)
    print(f"[attention] {dtype} {cache} {len(lens)} sequences, longest {max(lens)}", flush=True)
    _attend(cfg, lens, 2)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
def test_scales(dtype, cache, scale):
    """No weight to the scores, sharp ones (one position takes almost all), and a negative scale."""
    cfg = M.CacheConfig(2, 8, 2, 64, 32, 80, 40, dtype=dtype, cache_dtype=cache)
    _attend(cfg, [1111, 300], 3, scale)


def test_a_growing_maximum_and_scores_of_minus_infinity():
    """Scores that grow with the position, so that the running maximum moves at every step; keys of -infinity leave nothing."""
    cfg = M.CacheConfig(1, 4, 1, 64, 16, 100, 80, dtype=M.F32)
    q, table, lens, kp, vp, ks, vs = _filled(cfg, [1200], 4)
    q, kp = torch.ones_like(q).contiguous(), kp.clone()
    pos = torch.arange(80 * 16, device="cuda").reshape(80, 16).float()
    kp[table[0, :75].long()] = (pos[:75] * 0.05)[:, None, :, None].expand(75, 1, 16, 64).contiguous() / 64
    out, lse = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    ws = torch.zeros(max(16, M.mohge_cache_workspace_size(cfg)), dtype=torch.uint8, device="cuda")
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, None, None, 1.0, out, lse, ws)
    _check(cfg, q, table, lens, kp, vp, None, None, 1.0, out, lse)
    kp[...] = -math.inf
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, None, None, 1.0, out, lse, ws)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_pages_out_of_range_give_nan_and_touch_no_other_sequence(dtype, cache):
    cfg = M.CacheConfig(4, 8, 2, 128, 16, 400, 100, dtype=dtype, cache_dtype=cache)
    (q, table, lens, kp, vp, ks, vs), out, lse, ws = _attend(cfg, [500, 300, 1600, 7], 5)
    good = out.clone()
    for seq, col, page in ((0, 3, -1), (1, 18, 400), (2, 99, 1 << 30)):
        t = table.clone()
        t[seq, col] = page
        M.mohge_cache_attention(cfg, q, t, lens, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)
        others = [b for b in range(4) if b != seq]
        assert out[seq].isnan().all() and lse[seq].isnan().all() and torch.equal(out[others], good[others]), seq
    # longer than the table: NaN, and nothing past it is looked up
    long = lens.clone()
    long[2] = 1601
    M.mohge_cache_attention(cfg, q, table, long, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)
    assert out[2].isnan().all() and lse[2].isnan().all() and torch.equal(out[[0, 1, 3]], good[[0, 1, 3]])
    # a negative length is an empty sequence
    long[2] = -5
    M.mohge_cache_attention(cfg, q, table, long, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all() and torch.equal(out[[0, 1, 3]], good[[0, 1, 3]])


def test_counters_that_were_not_zero_leave_nan():
    cfg = M.CacheConfig(2, 8, 2, 128, 16, 800, 600)
    (q, table, lens, kp, vp, ks, vs), out, lse, ws = _attend(cfg, [9000, 40], 6)
    good = out.clone()
    ws[:16] = 77
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)
    assert out[0].isnan().all() and lse[0].isnan().all() and torch.equal(out[1], good[1])
    ws.zero_()
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)
    assert torch.equal(out, good)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_pages_past_32_bit_offsets(dtype, cache):
    """A cache of more than 2^31 elements; the sequence's pages are its last ones, written by the append."""
    kv, D, S, n = 8, 128, 128, 700
    n_pages = 2 ** 31 // (kv * D * S) + 64
    cfg = M.CacheConfig(1, 16, kv, D, S, n_pages, 8, dtype=dtype, cache_dtype=cache)
    t = torch.uint8 if cache == M.E4M3 else TYPES[cache]
    kp, vp = (torch.empty((n_pages, kv, S, D), dtype=t, device="cuda") for _ in range(2))
    ks, vs = (torch.empty((n_pages, kv, S), device="cuda") if cache == M.E4M3 else None for _ in range(2))
    table = torch.arange(n_pages - 1, n_pages - 9, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((n, kv, D), device="cuda").to(TYPES[dtype]) for _ in range(2))
    q = torch.randn((1, 16, D), device="cuda").to(TYPES[dtype])
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    print(f"[cache] {n_pages} pages", flush=True)
    M.mohge_cache_append(cfg, k, v, offsets, table, lens, kp, vp, ks, vs)
    pages = table[0, :-(-n // S)].long()
    for rows, store, scale in ((k, kp, ks), (v, vp, vs)):
        got = _values(store[pages], None if scale is None else scale[pages]).transpose(0, 1).reshape(kv, -1, D)[:, :n].transpose(0, 1)
        if scale is None:
            assert torch.equal(got, rows.double())
        else:
            assert ((got - rows.double()).abs() <= 2.0 ** -4 * rows.double().abs().amax(2, keepdim=True)).all()
    out, lse = torch.empty_like(q), torch.empty((1, 16), device="cuda")
    ws = torch.zeros(max(16, M.mohge_cache_workspace_size(cfg)), dtype=torch.uint8, device="cuda")
    M.mohge_cache_attention(cfg, q, table, lens, kp, vp, ks, vs, D ** -0.5, out, lse, ws)
    _check(cfg, q, table, lens, kp, vp, ks, vs, D ** -0.5, out, lse)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("head,page,kv", [(64, 16, 3), (128, 64, 1), (256, 256, 2)])
def test_append(dtype, cache, head, page, kv):
    """Rows of several sequences, none for some, from slices of wider rows; everything else in the pages stays as it was."""
    new, past = [5, 0, 1, 300, 0, 17, 2 * page], [0, 3, page - 1, 7, 0, 2 * page, 40]
    lens = [a + b for a, b in zip(new, past)]
    columns = max(-(-n // page) for n in lens) + 1
    n_pages = sum(-(-n // page) for n in lens) + 3
    cfg = M.CacheConfig(len(new), kv, kv, head, page, n_pages, columns, dtype=dtype, cache_dtype=cache)
    gen = torch.Generator(device="cuda").manual_seed(head + page)
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    table = torch.full((len(new), columns), -7, dtype=torch.int32)
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            table[b, i] = order.pop()
    T, W = sum(new), kv * head
    wide = torch.randn((T, 3 * W + 24), generator=gen, device="cuda").to(TYPES[dtype])
    wide[1] *= 1e-3
    wide[2] = 0
    k, v = wide[:, 8:8 + W].view(T, kv, head), wide[:, 16 + 2 * W:16 + 3 * W].view(T, kv, head)
    g = GuardBands()
    t = torch.uint8 if cache == M.E4M3 else TYPES[cache]
    stores = [g.wrap(torch.empty((n_pages, kv, page, head), dtype=t, device="cuda"), n).fill_(5) for n in ("k_pages", "v_pages")]
    scales = [g.wrap(torch.empty((n_pages, kv, page), device="cuda"), n).fill_(9.0) if cache == M.E4M3 else None for n in ("k_scale", "v_scale")]
    offsets = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    M.mohge_cache_append(cfg, k, v, offsets, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), *stores, *scales)
    written = torch.zeros((n_pages, page), dtype=torch.bool, device="cuda")
    for rows, store, scale in ((k, stores[0], scales[0]), (v, stores[1], scales[1])):
        i = 0
        for b, n in enumerate(new):
            for p in range(past[b], lens[b]):
                at, off = int(table[b, p // page]), p % page
                written[at, off] = True
                want = rows[i].double()
                if scale is None:
                    assert torch.equal(store[at, :, off], rows[i]), (b, p)
                else:
                    top = want.abs().amax(1)
                    ws = torch.where(top > 0, top / 448, torch.ones_like(top))
                    assert ((scale[at, :, off].double() - ws).abs() <= 4 * U * ws).all()
                    got = store[at, :, off].view(torch.float8_e4m3fn).double() * scale[at, :, off].double()[:, None]
                    bound = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * ws[:, None]) + 8 * U * want.abs()
                    assert ((got - want).abs() <= bound).all(), (b, p)
                i += 1
        rest = ~written[:, None, :, None].expand(store.shape)
        assert (store[rest] == 5).all() and (scale is None or (scale[rest[..., 0]] == 9.0).all())
    g.check()


def test_append_leaves_out_what_has_no_place():
    cfg = M.CacheConfig(4, 2, 2, 64, 16, 6, 2)
    k = torch.randn((4, 2, 64), device="cuda").bfloat16()
    kp, vp = (torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[0, 1], [2, 6], [-1, 3], [4, 5]], dtype=torch.int32, device="cuda")
    # fits; page 6 of 6; page -1; past the table
    lens = torch.tensor([17, 20, 3, 33], dtype=torch.int32, device="cuda")
    M.mohge_cache_append(cfg, k, k, None, table, lens, kp, vp)
    want = torch.zeros_like(kp)
    want[1, :, 0] = k[0]
    assert torch.equal(kp, want) and torch.equal(vp, want)
    # a sequence that sits the step out
    M.mohge_cache_append(cfg, k, k, None, table, torch.zeros_like(lens), kp, vp)
    assert torch.equal(kp, want)
    # rows that no sequence has
    M.mohge_cache_append(cfg, k, k, torch.tensor([0, 0, 0, 0, 1], dtype=torch.int32, device="cuda"), table, torch.full_like(lens, 5), kp, vp)
    want[4, :, 4] = k[0]
    assert torch.equal(kp, want)


def test_same_bits_every_time_on_any_stream_and_in_a_graph_whose_lengths_change():
    cfg = M.CacheConfig(3, 8, 2, 128, 16, 900, 400, cache_dtype=M.E4M3)
    kv = M.KVCache(cfg)
    gen = torch.Generator(device="cuda").manual_seed(8)
    draw = lambda n, h: torch.randn((n, h, 128), generator=gen, device="cuda").bfloat16()  # noqa: E731
    kv.grow([5000, 1, 260])
    k, v = draw(5261, 2), draw(5261, 2)
    kv.append(k, v, torch.tensor([0, 5000, 5001, 5261], dtype=torch.int32, device="cuda"))
    q, k1, v1 = draw(3, 8), draw(3, 2), draw(3, 2)

    def step():
        kv.append(k1, v1)
        kv.attend(q)

    def results():
        torch.cuda.synchronize()
        return kv.out.clone(), kv.lse.clone()

    kv.grow([1, 1, 1])
    step()
    want = results()
    step()                                          # the same rows in the same places
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(20):
        kv.grow([1, 30, 16])
        for t in (q, k1, v1):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        step()
        eager = results()
        kv.out.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), eager)), i
    for b, n in enumerate(kv.lengths):
        assert kv.seq_lens[b] == n


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16])
@pytest.mark.parametrize("dtype,cache", KINDS)
def test_many_parts_for_every_number_of_heads(group, dtype, cache):
    """Rows that more than a dozen workgroups share, where heads leave lanes over for parts."""
    cfg = M.CacheConfig(2, 2 * group, 2, 64, 16, 700, 600, dtype=dtype, cache_dtype=cache)
    _attend(cfg, [9001, 77], 11)
