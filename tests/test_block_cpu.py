"""The operators around the layer, host side: what mohge_block.h declares, argument checks, the 4-bit quantiser,
the handing out of pages."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2604_23108_amd as M
from paper_2604_23108_amd import block_binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = C.c_void_p(256)                     # an aligned address that no refused call touches
ODD = C.c_void_p(264)


def test_library_exports_what_the_header_declares():
    header = open(os.path.join(ROOT, "include", "mohge_block.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(mohge_[a-z_0-9]+)\s*\(", header))
    assert declared == set(B.EXPORTS) == set(B._ARGS)
    for name in declared:
        assert hasattr(M.lib(), name) and hasattr(M, name), name
    assert int(re.search(r"MOHGE_E4M3\s*=\s*(\d+)", header).group(1)) == M.E4M3
    assert (C.sizeof(B._CNorm), C.sizeof(B._CCache), C.sizeof(B._CProj)) == (20, 36, 24)


def _refused(code, text):
    def check(rc):
        assert rc == code and text in M.mohge_last_error(), (rc, M.mohge_last_error())
    return check


@pytest.mark.parametrize("kw,msg", [(dict(T=-1), "T = -1"), (dict(T=(1 << 21) + 1), "T = "), (dict(d=12), "d = 12"), (dict(d=0), "d = 0"),
                                    (dict(d=32776), "d = "), (dict(dtype=M.E4M3), "dtype = 2"), (dict(y_dtype=M.F32), "y_dtype"),
                                    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps")])
def test_norm_configurations_are_refused(kw, msg):
    cfg = M.NormConfig(**{**dict(T=4, d=64), **kw})
    f, g = B._call("mohge_rmsnorm"), B._call("mohge_rmsnorm_bwd")
    _refused(-1, msg)(f(cfg.ref, *[None] * 8))
    _refused(-1, msg)(g(cfg.ref, *[None] * 8, 0, None))
    assert M.mohge_norm_workspace_size(cfg) == 0


def test_norm_pointers_are_checked():
    f, g = B._call("mohge_rmsnorm"), B._call("mohge_rmsnorm_bwd")
    cfg, q8 = M.NormConfig(4, 64), M.NormConfig(4, 64, y_dtype=M.E4M3)
    _refused(-2, "cfg")(f(None, *[None] * 8))
    _refused(-2, "x is NULL")(f(cfg.ref, None, None, P, None, P, None, None, None))
    _refused(-2, "weight is NULL")(f(cfg.ref, P, None, None, None, P, None, None, None))
    _refused(-2, "y is NULL")(f(cfg.ref, P, None, P, None, None, None, None, None))
    _refused(-3, "residual")(f(cfg.ref, P, ODD, P, None, P, None, None, None))
    _refused(-2, "y_scale is NULL")(f(q8.ref, P, None, P, None, P, None, None, None))
    _refused(-1, "y_scale given")(f(cfg.ref, P, None, P, None, P, P, None, None))
    n = M.mohge_norm_workspace_size(cfg)
    assert n > 0 and n == M.mohge_norm_workspace_size(M.NormConfig(100000, 64))
    _refused(-4, "workspace")(g(cfg.ref, P, P, P, P, None, P, P, P, n - 1, None))
    _refused(-2, "rstd is NULL")(g(cfg.ref, P, P, P, None, None, P, P, P, n, None))
    _refused(-2, "dweight is NULL")(g(cfg.ref, P, P, P, P, None, P, None, P, n, None))
    assert f(M.NormConfig(0, 64).ref, *[None] * 8) == 0          # nothing to do


_CACHE = dict(n_seqs=2, n_heads=8, n_kv_heads=2, head_size=64, page_size=16, n_pages=10, max_pages=4)


@pytest.mark.parametrize("kw,msg", [(dict(n_seqs=-1), "n_seqs"), (dict(n_heads=7), "n_heads"), (dict(n_kv_heads=0), "n_heads"),
                                    (dict(n_heads=2048, n_kv_heads=2048), "n_heads"), (dict(n_seqs=1 << 22), "2^24"),
                                    (dict(head_size=96), "head_size"), (dict(page_size=8), "page_size"),
                                    (dict(page_size=48), "page_size"), (dict(page_size=512), "page_size"),
                                    (dict(n_pages=0), "positive"), (dict(max_pages=0), "positive"),
                                    (dict(max_pages=1 << 27), "int32"), (dict(dtype=M.E4M3), "dtype"),
                                    (dict(cache_dtype=M.F32), "cache_dtype"), (dict(dtype=M.F32, cache_dtype=M.E4M3), "cache_dtype")])
def test_cache_configurations_are_refused(kw, msg):
    cfg = M.CacheConfig(**{**_CACHE, **kw})
    _refused(-1, msg)(B._call("mohge_cache_append")(cfg.ref, 0, None, 0, None, 0, *[None] * 8))
    _refused(-1, msg)(B._call("mohge_cache_attention")(cfg.ref, None, 0, *[None] * 6, 1.0, None, None, None, 0, None))
    assert M.mohge_cache_workspace_size(cfg) == 0


def test_cache_arguments_are_checked():
    cfg, e8 = M.CacheConfig(**_CACHE), M.CacheConfig(**_CACHE, cache_dtype=M.E4M3)
    f, g = B._call("mohge_cache_append"), B._call("mohge_cache_attention")

    def append(c=cfg, n=2, k=P, ks=128, v=P, vs=128, off=None, table=P, lens=P, kp=P, vp=P, s=None, t=None):
        return f(c.ref, n, k, ks, v, vs, off, table, lens, kp, vp, s, t, None)

    _refused(-1, "n_tokens = -1")(append(n=-1))
    _refused(-1, "without tok_offsets")(append(n=3))
    _refused(-1, "2^34")(append(n=1 << 30, off=P))
    _refused(-2, "k is NULL")(append(k=None))
    _refused(-2, "v is NULL")(append(v=None))
    _refused(-3, "tok_offsets")(append(off=ODD))
    _refused(-2, "block_table is NULL")(append(table=None))
    _refused(-3, "k_pages")(append(kp=ODD))
    _refused(-1, "k_stride")(append(ks=120))
    _refused(-3, "v_stride")(append(vs=132))
    _refused(-2, "k_scale is NULL")(append(c=e8))
    _refused(-1, "without scales")(append(s=P, t=P))
    assert append(n=0, off=P, k=None) == 0
    ws = max(16, M.mohge_cache_workspace_size(cfg))

    def attend(c=cfg, q=P, qs=512, table=P, lens=P, kp=P, vp=P, s=None, t=None, out=P, lse=None, w=P, n=ws):
        return g(c.ref, q, qs, table, lens, kp, vp, s, t, 0.125, out, lse, w, n, None)

    _refused(-2, "q is NULL")(attend(q=None))
    _refused(-2, "out is NULL")(attend(out=None))
    _refused(-3, "lse")(attend(lse=ODD))
    _refused(-2, "workspace is NULL")(attend(w=None))
    _refused(-2, "seq_lens is NULL")(attend(lens=None))
    _refused(-1, "q_stride")(attend(qs=504))
    _refused(-3, "q_stride")(attend(qs=516))
    _refused(-2, "k_scale is NULL")(attend(c=e8))
    long = M.CacheConfig(**{**_CACHE, "max_pages": 100000})
    need = M.mohge_cache_workspace_size(long)
    assert need > 0
    _refused(-4, "workspace")(attend(c=long, n=need - 1))
    assert attend(c=M.CacheConfig(**{**_CACHE, "n_seqs": 0}), q=None) == 0


@pytest.mark.parametrize("kw,msg", [(dict(T=-1), "T = -1"), (dict(T=33), "T = 33"), (dict(n_in=96), "n_in"), (dict(n_in=0), "n_in"),
                                    (dict(n_out=0), "n_out"), (dict(group=16), "group"), (dict(group=0), "group"),
                                    (dict(x_dtype=M.F32), "x_dtype"), (dict(y_dtype=M.E4M3), "y_dtype")])
def test_projections_are_refused(kw, msg):
    cfg = M.ProjConfig(**{**dict(T=2, n_in=256, n_out=64, group=64), **kw})
    _refused(-1, msg)(B._call("mohge_proj_w4")(cfg.ref, *[None] * 7))


def test_projection_pointers_are_checked():
    f = B._call("mohge_proj_w4")
    cfg, e8 = M.ProjConfig(2, 256, 64), M.ProjConfig(2, 256, 64, x_dtype=M.E4M3)
    _refused(-2, "x is NULL")(f(cfg.ref, None, None, P, P, None, P, None))
    _refused(-2, "codes is NULL")(f(cfg.ref, P, None, None, P, None, P, None))
    _refused(-2, "scales is NULL")(f(cfg.ref, P, None, P, None, None, P, None))
    _refused(-3, "zeros")(f(cfg.ref, P, None, P, P, ODD, P, None))
    _refused(-2, "y is NULL")(f(cfg.ref, P, None, P, P, None, None, None))
    _refused(-2, "x_scale is NULL")(f(e8.ref, P, None, P, P, None, P, None))
    _refused(-1, "x_scale given")(f(cfg.ref, P, P, P, P, None, P, None))
    assert f(M.ProjConfig(0, 256, 64).ref, *[None] * 7) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros(4, 64)
    with pytest.raises(M.MohgeError, match="y: "):
        M.mohge_rmsnorm(M.NormConfig(4, 64, dtype=M.F32), None, None, None, None, t[:, :32])
    with pytest.raises(M.MohgeError, match="GPU"):
        M.mohge_rmsnorm(M.NormConfig(4, 64, dtype=M.F32), t, None, None, None, None)
    with pytest.raises(M.MohgeError, match="x: .*bfloat16 needed"):
        M.mohge_proj_w4(M.ProjConfig(4, 64, 8, group=32), t, None, None, None, None, None)
    with pytest.raises(M.MohgeError, match="q: "):
        M.mohge_cache_attention(M.CacheConfig(**_CACHE), t, None, None, None, None, None, None, 1.0, None, None, None)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_w4(group, zeros):
    gen = torch.Generator().manual_seed(group)
    w = torch.randn(6, 384, generator=gen) * torch.exp(torch.randn(6, 1, generator=gen))
    w[0, :group] = 0.0                                      # a group of zeros
    w[1, :group] = 3.5                                      # all of one sign
    w[2, :group] = -w[2, :group].abs()
    codes, scales, z = M.quantize_w4(w, group, zeros)
    assert codes.shape == (6, 192) and scales.shape == (6, 384 // group) and scales.dtype == torch.bfloat16
    assert (z is not None) == zeros
    c = torch.stack([codes & 15, codes >> 4], 2).reshape(6, 384 // group, group).double()
    s = scales.double().unsqueeze(2)
    back = s * (c - (z.double().unsqueeze(2) if zeros else 8.0))
    # half a step, or what the bf16 rounding of the scale (2^-9) and of the zero point leave outside the codes' range
    blk = w.double().reshape(6, -1, group)
    assert ((back - blk).abs() <= s * (0.5 + (0.5 if zeros else 0.0) + 15 * 2.0 ** -8) + 1e-12).all()
    assert (back[0, 0] == 0).all()
    with pytest.raises(ValueError, match="multiple"):
        M.quantize_w4(w[:, :100], group)


def test_pages_are_handed_out_and_taken_back():
    cfg = M.CacheConfig(n_seqs=3, n_heads=4, n_kv_heads=2, head_size=64, page_size=16, n_pages=8, max_pages=4)
    kv = M.KVCache(cfg, device="cpu")
    kv.grow([17, 0, 16])
    assert kv.seq_lens.tolist() == [17, 0, 16] and [len(p) for p in kv.pages] == [2, 0, 1]
    kv.grow([1, 1, 1])
    assert kv.seq_lens.tolist() == [18, 1, 17] and [len(p) for p in kv.pages] == [2, 1, 2]
    for b, pages in enumerate(kv.pages):
        assert kv.block_table[b].tolist() == pages + [-1] * (4 - len(pages))
    assert len({p for pages in kv.pages for p in pages}) == 5
    before = (list(kv.lengths), kv.block_table.clone())
    with pytest.raises(M.MohgeError, match="4 pages needed, 3 free"):
        kv.grow([31, 16, 20])
    with pytest.raises(M.MohgeError, match="max_pages"):
        kv.grow([47, 0, 0])
    with pytest.raises(M.MohgeError, match="count for each"):
        kv.grow([1, 1])
    with pytest.raises(M.MohgeError, match="count for each"):
        kv.grow([1, -1, 0])
    assert kv.lengths == before[0] and torch.equal(kv.block_table, before[1])
    kv.free(0)
    assert kv.seq_lens.tolist() == [0, 1, 17] and kv.block_table[0].tolist() == [-1] * 4
    kv.grow([64, 0, 0])
    assert len(kv.pages[0]) == 4 and len({p for pages in kv.pages for p in pages}) == 7


def test_positions_leave_room_for_rounding_up():
    """Lengths are rounded up to a unit of the attention in int32: a table for 2^31 - 16 positions would overflow there."""
    one = dict(n_seqs=1, n_heads=1, n_kv_heads=1, head_size=64, page_size=16, n_pages=10)
    assert M.mohge_cache_workspace_size(M.CacheConfig(**one, max_pages=1 << 26)) > 0
    for pages in ((1 << 26) + 1, (1 << 27) - 1):
        assert M.mohge_cache_workspace_size(M.CacheConfig(**one, max_pages=pages)) == 0
        assert "int32" in M.mohge_last_error()
