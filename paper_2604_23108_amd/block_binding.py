"""Binding of the operators around the layer (`include/mohge_block.h`, in libmohge.so): argument marshalling only, with
the names and argument order of the header, plus objects that hold the buffers of one use (`ResidualNorm`, `KVCache`,
`ProjW4`).

Tensors must live on the GPU and be contiguous (the rows of q, k and v may be further apart); the current torch
stream is passed as the HIP stream.  The calls of a step go through the extension module `_block_native`
(`csrc/block_py.cpp`), the rest through ctypes.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from typing import Optional, Sequence

import torch

from .binding import BF16, F32, MohgeError, lib

E4M3 = 2

EXPORTS = ["mohge_rmsnorm", "mohge_rmsnorm_bwd", "mohge_norm_workspace_size", "mohge_cache_append",
           "mohge_cache_attention", "mohge_cache_workspace_size", "mohge_proj_w4"]

# argument kinds: P pointer, I int32, L int64, F float, Z size_t
_ARGS = {"mohge_rmsnorm": "P" * 9, "mohge_rmsnorm_bwd": "P" * 9 + "ZP", "mohge_norm_workspace_size": "P",
         "mohge_cache_append": "PIPLPL" + "P" * 8, "mohge_cache_attention": "PPL" + "P" * 6 + "FPPPZP",
         "mohge_cache_workspace_size": "P", "mohge_proj_w4": "P" * 8}
_KINDS = {"P": C.c_void_p, "I": C.c_int32, "L": C.c_int64, "F": C.c_float, "Z": C.c_size_t}

_calls = {}


def _call(name):
    """The function with its argument types declared (an object of its own: lib()'s stay as they are)."""
    f = _calls.get(name)
    if f is None:
        f = lib()[name]
        f.restype = C.c_size_t if name.endswith("_size") else C.c_int
        f.argtypes = [_KINDS[k] for k in _ARGS[name]]
        _calls[name] = f
    return f


class _Native:
    """The extension module, loaded and given the library's entry points at the first call."""

    CALLS = ("rmsnorm", "rmsnorm_bwd", "cache_append", "cache_attention", "proj_w4")

    def __getattr__(self, name):
        if name not in self.CALLS and name != "file":
            raise AttributeError(f"_block_native has no {name}")
        from .build import native_path
        path = native_path(torch.__version__)
        if not os.path.exists(path):
            raise MohgeError(f"{path} is missing: build it with `python -m paper_2604_23108_amd.build` (there is no fallback path)")
        spec = importlib.util.spec_from_file_location("_block_native", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        entries = [f"mohge_{n}" for n in self.CALLS + ("last_error",)]
        module.bind(MohgeError, *[C.cast(getattr(lib(), e), C.c_void_p).value for e in entries])
        for n in self.CALLS:
            setattr(self, n, getattr(module, n))
        self.file = path
        return self.__dict__[name]


_native = _Native()


class _CNorm(C.Structure):
    _fields_ = [("T", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("y_dtype", C.c_int32), ("eps", C.c_float)]


class _CCache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_heads", "n_kv_heads", "head_size", "page_size", "n_pages",
                                         "max_pages", "dtype", "cache_dtype")]


class _CProj(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "n_in", "n_out", "group", "x_dtype", "y_dtype")]


_TORCH = {BF16: torch.bfloat16, F32: torch.float32, E4M3: torch.uint8}


def torch_type(dtype: int) -> torch.dtype:
    """The torch type that holds BF16, F32 or E4M3 (codes: one byte each)."""
    if dtype not in _TORCH:
        raise MohgeError(f"dtype {dtype} unknown")
    return _TORCH[dtype]


class NormConfig:
    """Python mirror of `mohge_norm_config`."""

    def __init__(self, T: int, d: int, dtype: int = BF16, y_dtype: Optional[int] = None, eps: float = 1e-6):
        self.T, self.d, self.dtype, self.eps = T, d, dtype, eps
        self.y_dtype = dtype if y_dtype is None else y_dtype
        self._c = _CNorm(T, d, dtype, self.y_dtype, eps)
        self.ref = C.addressof(self._c)


class CacheConfig:
    """Python mirror of `mohge_cache_config`."""

    def __init__(self, n_seqs: int, n_heads: int, n_kv_heads: int, head_size: int, page_size: int, n_pages: int,
                 max_pages: int, dtype: int = BF16, cache_dtype: Optional[int] = None):
        self.n_seqs, self.n_heads, self.n_kv_heads, self.head_size = n_seqs, n_heads, n_kv_heads, head_size
        self.page_size, self.n_pages, self.max_pages, self.dtype = page_size, n_pages, max_pages, dtype
        self.cache_dtype = dtype if cache_dtype is None else cache_dtype
        self._c = _CCache(n_seqs, n_heads, n_kv_heads, head_size, page_size, n_pages, max_pages, dtype, self.cache_dtype)
        self.ref = C.addressof(self._c)


class ProjConfig:
    """Python mirror of `mohge_proj_config`."""

    def __init__(self, T: int, n_in: int, n_out: int, group: int = 128, x_dtype: int = BF16, y_dtype: int = BF16):
        self.T, self.n_in, self.n_out, self.group, self.x_dtype, self.y_dtype = T, n_in, n_out, group, x_dtype, y_dtype
        self._c = _CProj(T, n_in, n_out, group, x_dtype, y_dtype)
        self.ref = C.addressof(self._c)


def mohge_rmsnorm(cfg: NormConfig, x, residual, weight, sum_out, y, y_scale=None, rstd=None):
    _native.rmsnorm(cfg.ref, x, residual, weight, sum_out, y, y_scale, rstd)


def mohge_norm_workspace_size(cfg: NormConfig) -> int:
    return int(_call("mohge_norm_workspace_size")(cfg.ref))


def mohge_rmsnorm_bwd(cfg: NormConfig, dy, h, weight, rstd, dsum, dx, dweight, workspace):
    _native.rmsnorm_bwd(cfg.ref, dy, h, weight, rstd, dsum, dx, dweight, workspace)


def mohge_cache_append(cfg: CacheConfig, k, v, tok_offsets, block_table, seq_lens, k_pages, v_pages, k_scale=None,
                       v_scale=None):
    _native.cache_append(cfg.ref, k, v, tok_offsets, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale)


def mohge_cache_workspace_size(cfg: CacheConfig) -> int:
    return int(_call("mohge_cache_workspace_size")(cfg.ref))


def mohge_cache_attention(cfg: CacheConfig, q, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale, scale: float,
                          out, lse, workspace):
    _native.cache_attention(cfg.ref, q, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale, scale, out, lse, workspace)


def mohge_proj_w4(cfg: ProjConfig, x, x_scale, codes, scales, zeros, y):
    _native.proj_w4(cfg.ref, x, x_scale, codes, scales, zeros, y)


class ResidualNorm:
    """The norm in front of a layer: output buffers, and for training the gradients' (made once)."""

    def __init__(self, cfg: NormConfig, weight: torch.Tensor, backward: bool = False):
        self.cfg, self.weight, self.has_backward = cfg, weight, backward
        dev = dict(device=weight.device)
        shape, t = (cfg.T, cfg.d), torch_type(cfg.dtype)
        self.sum = torch.empty(shape, dtype=t, **dev)
        self.y = torch.empty(shape, dtype=torch_type(cfg.y_dtype), **dev)
        self.y_scale = torch.empty(cfg.T, dtype=torch.float32, **dev) if cfg.y_dtype == E4M3 else None
        self.rstd = torch.empty(cfg.T, dtype=torch.float32, **dev)
        self._h = None
        if backward:
            if cfg.y_dtype == E4M3:
                raise MohgeError("backward needs an output in the type of x")
            self.dx, self.dweight = torch.empty(shape, dtype=t, **dev), torch.empty(cfg.d, dtype=torch.float32, **dev)
            self.ws = torch.empty(max(16, mohge_norm_workspace_size(cfg)), dtype=torch.uint8, **dev)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """y; the new residual stream is left in `sum` (without a residual it is x itself, which `backward` then reads again)."""
        out = None if residual is None else self.sum
        mohge_rmsnorm(self.cfg, x, residual, self.weight, out, self.y, self.y_scale, self.rstd)
        self._h = x if residual is None else self.sum
        return self.y

    def backward(self, dy: torch.Tensor, dsum: Optional[torch.Tensor] = None) -> torch.Tensor:
        """After `forward`: the gradient of x (and of residual), with `dsum` the one that reaches the residual stream
        past the norm; the weight's is left in `dweight`."""
        if not self.has_backward or self._h is None:
            raise MohgeError("backward needs a norm created with backward=True and its forward pass")
        mohge_rmsnorm_bwd(self.cfg, dy, self._h, self.weight, self.rstd, dsum, self.dx, self.dweight, self.ws)
        return self.dx


class KVCache:
    """Pages of keys and values, which sequence has which, and how long each sequence is.

    The page numbers are handed out on the host: `grow` gives every sequence the pages that its new positions need and
    sets the lengths, `append` writes their keys and values, `attend` reads.  `free` gives a sequence's pages back.  The tensors
    stay the same ones, so that recorded calls see what `grow` and `free` change.
    """

    def __init__(self, cfg: CacheConfig, device="cuda"):
        self.cfg = cfg
        pages, t = (cfg.n_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_size), torch_type(cfg.cache_dtype)
        self.k_pages, self.v_pages = (torch.zeros(pages, dtype=t, device=device) for _ in range(2))
        scales = cfg.cache_dtype == E4M3
        self.k_scale, self.v_scale = (torch.ones(pages[:3], device=device) if scales else None for _ in range(2))
        self.block_table = torch.full((cfg.n_seqs, cfg.max_pages), -1, dtype=torch.int32, device=device)
        # the lengths, and those of the sequences that the last `grow` made longer (0: the others); rows start 16 bytes apart
        self._lens = torch.zeros((2, -(-cfg.n_seqs // 4) * 4), dtype=torch.int32, device=device)
        self.seq_lens, self._grown = (row[:cfg.n_seqs] for row in self._lens)
        self._all_grew = True
        self.out = torch.empty((cfg.n_seqs, cfg.n_heads, cfg.head_size), dtype=torch_type(cfg.dtype), device=device)
        self.lse = torch.empty((cfg.n_seqs, cfg.n_heads), dtype=torch.float32, device=device)
        self.ws = torch.zeros(max(16, mohge_cache_workspace_size(cfg)), dtype=torch.uint8, device=device)
        self.lengths = [0] * cfg.n_seqs
        self.pages = [[] for _ in range(cfg.n_seqs)]
        self._unused = list(range(cfg.n_pages - 1, -1, -1))

    def grow(self, new: Sequence[int]):
        """`new[b]` further positions for every sequence; raises, and changes nothing, where there is no room."""
        c = self.cfg
        if len(new) != c.n_seqs or any(n < 0 for n in new):
            raise MohgeError(f"grow takes a count for each of {c.n_seqs} sequences")
        lengths = [a + n for a, n in zip(self.lengths, new)]
        more = [-(-n // c.page_size) - len(p) for n, p in zip(lengths, self.pages)]
        if sum(more) > len(self._unused):
            raise MohgeError(f"{sum(more)} pages needed, {len(self._unused)} free")
        if any(-(-n // c.page_size) > c.max_pages for n in lengths):
            raise MohgeError(f"a sequence would need more than max_pages = {c.max_pages} pages")
        self.lengths = lengths
        if any(more):
            rows, cols, pages = [], [], []
            for b, n in enumerate(more):
                for _ in range(n):
                    rows.append(b)
                    cols.append(len(self.pages[b]))
                    self.pages[b].append(self._unused.pop())
                    pages.append(self.pages[b][-1])
            at = torch.tensor([rows, cols, pages], device=self.block_table.device)
            self.block_table[at[0], at[1]] = at[2].int()
        all_grew, had = all(n or not length for n, length in zip(new, lengths)), self._all_grew
        self._all_grew = all_grew
        if had and all_grew and len(set(new)) == 1:
            self._lens += new[0]                           # the rows are equal and stay so
        else:
            counts = torch.tensor(list(new), dtype=torch.int32, device=self._lens.device)
            self.seq_lens += counts
            self._grown.copy_(self.seq_lens * (counts > 0))

    def free(self, seq: int):
        """The sequence is empty again, its pages are handed out anew."""
        self._unused += reversed(self.pages[seq])
        self.pages[seq], self.lengths[seq] = [], 0
        self.block_table[seq] = -1
        self.seq_lens[seq] = self._grown[seq] = 0

    def append(self, k: torch.Tensor, v: torch.Tensor, tok_offsets: Optional[torch.Tensor] = None):
        """Keys and values of the positions that the last `grow` added: rows tok_offsets[b] .. of k and v for sequence b, or one
        row for every sequence, its last position; there the rows of sequences that did not grow are left out."""
        lens = self._grown if tok_offsets is None else self.seq_lens
        mohge_cache_append(self.cfg, k, v, tok_offsets, self.block_table, lens, self.k_pages, self.v_pages, self.k_scale, self.v_scale)

    def attend(self, q: torch.Tensor, scale: Optional[float] = None) -> torch.Tensor:
        """Attention of one query row per sequence over all its positions (scale: 1 / sqrt(head_size) unless given)."""
        mohge_cache_attention(self.cfg, q, self.block_table, self.seq_lens, self.k_pages, self.v_pages, self.k_scale,
                              self.v_scale, self.cfg.head_size ** -0.5 if scale is None else scale, self.out, self.lse, self.ws)
        return self.out


class ProjW4:
    """A projection with 4-bit weights (`quantize_w4`) and its output buffer."""

    def __init__(self, cfg: ProjConfig, codes: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor] = None):
        self.cfg, self.codes, self.scales, self.zeros = cfg, codes, scales, zeros
        self.y = torch.empty((cfg.T, cfg.n_out), dtype=torch_type(cfg.y_dtype), device=codes.device)

    def forward(self, x: torch.Tensor, x_scale: Optional[torch.Tensor] = None) -> torch.Tensor:
        mohge_proj_w4(self.cfg, x, x_scale, self.codes, self.scales, self.zeros, self.y)
        return self.y
