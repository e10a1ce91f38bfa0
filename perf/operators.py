"""The operators of a decoder block around the MoHGE layer, as cases that can be timed and compared.

A case is one call of one operator: the root-mean-square norm with the residual's addition (`norm`,
and its backward pass `norm_bwd`), new keys and values into a paged cache (`append`), attention of one
new token per sequence over that cache (`attention`), and the product with 4-bit weights of a decode
step's projections (`proj`).  `listed()` names cases from the smallest call to the largest, `draw()`
gives further ones of the same ranges.  With `own` false, `run` computes the operator in elementary
torch operations in 32 bits; with `own` true it makes the framework's calls.

Hidden sizes are those of `synth.WORKLOADS` and the layer tests plus odd ones; heads, pages and lengths are
generic.  Inputs are drawn on the GPU: activations, keys and values ~ N(0, 1), 4-bit codes uniform with
scales around 0.02 / 4.6, lengths of a batch spread evenly from the shortest to the longest.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _norm(T, d, **kw):
    return dict(dict(op="norm", T=T, d=d, dtype="bf16", y="same", residual=True), **kw)


def _norm_bwd(T, d, **kw):
    return dict(dict(op="norm_bwd", T=T, d=d, dtype="bf16", dsum=True), **kw)


def _append(seqs, tokens, **kw):
    """`tokens` new ones in all, over the sequences (0: one each)."""
    return dict(dict(op="append", seqs=seqs, tokens=tokens, past=500, heads=32, kv_heads=8, head=128, page=16, dtype="bf16",
                     cache="same"), **kw)


def _attention(seqs, shortest, longest, **kw):
    return dict(dict(op="attention", seqs=seqs, shortest=shortest, longest=longest, heads=32, kv_heads=8, head=128, page=16,
                     dtype="bf16", cache="same"), **kw)


def _proj(T, n_in, n_out, **kw):
    return dict(dict(op="proj", T=T, n_in=n_in, n_out=n_out, group=128, zeros=False, x="bf16", y="bf16"), **kw)


def listed():
    return [
        # interactive decoding: the norm in front of the layer for one token, where latency counts
        dict(_norm(1, 4096), name="norm_1"),
        # a batch of odd size whose rows go on as 8-bit codes
        dict(_norm(777, 1344, y="e4m3"), name="norm_777_8bit"),
        # the largest prefill
        dict(_norm(16384, 4096), name="norm_16384"),
        # training in fp32, as one runs it to check a model's numerics, odd number of tokens
        dict(_norm_bwd(777, 1024, dtype="f32"), name="norm_bwd_777_f32"),
        # a full micro-batch of training, the gradient of the residual path added
        dict(_norm_bwd(8192, 2048), name="norm_bwd_8192"),
        # a decode step of 32 sequences: one token each into the cache
        dict(_append(32, 0), name="append_32"),
        # prompts of uneven length (short ones that end inside a page among them) into an 8-bit cache
        dict(_append(5, 9003, past=0, page=64, cache="e4m3"), name="append_9003_8bit"),
        # interactive decoding with a short context: latency
        dict(_attention(1, 1531, 1531, heads=16, kv_heads=4, head=64), name="attention_1"),
        # a decode step of a server's batch: lengths from empty to long
        dict(_attention(32, 0, 8191), name="attention_32_ragged"),
        # two very long contexts in 8 bits: few rows, a long axis
        dict(_attention(2, 100000, 131072, page=64, cache="e4m3"), name="attention_2_long_8bit"),
        # the query, key and value projections of one token
        dict(_proj(1, 4096, 6144), name="proj_1"),
        # logits of a batch in fp32, from 8-bit rows, finer groups with zero points, an odd number of outputs
        dict(_proj(32, 4096, 65001, group=64, zeros=True, x="e4m3", y="f32"), name="proj_32_logits"),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_bwd", "append", "attention", "attention", "attention", "proj", "proj"])
    if op in ("norm", "norm_bwd"):
        T = _log_int(rng, 1, 16384) | 1
        d = rng.choice([1024, 1344, 2048, 2560, 4096, 8 * (_log_int(rng, 16, 1024) | 1)])
        if op == "norm":
            c = _norm(T, d, dtype=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["same", "same", "e4m3"]),
                      residual=rng.random() < 0.7)
        else:
            c = _norm_bwd(T, d, dtype=rng.choice(["bf16", "bf16", "f32"]), dsum=rng.random() < 0.7)
    elif op == "proj":
        n_in, group = rng.choice([(1024, 128), (1024, 32), (1344, 64), (1344, 32), (2048, 128), (2560, 64), (4096, 128), (4096, 32),
                                  (8192, 128)])
        c = _proj(rng.randint(1, 32), n_in, _log_int(rng, 256, 65000) | 1 if rng.random() < 0.5 else rng.choice([1024, 2048, 4096, 6144, 32768]),
                  group=group, zeros=rng.random() < 0.5, x=rng.choice(["bf16", "bf16", "e4m3"]), y=rng.choice(["bf16", "bf16", "f32"]))
    else:
        head, kv = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8, 8, 16])
        dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kw = dict(heads=kv * rng.choice([1, 2, 4, 4, 7, 8, 16]), kv_heads=kv, head=head, page=rng.choice([16, 32, 64, 128]), dtype=dt,
                  cache=rng.choice(["same", "e4m3"]) if dt == "bf16" else "same")
        seqs = _log_int(rng, 1, 128)
        if op == "append":
            if rng.random() < 0.5:
                c = _append(seqs, 0, past=_log_int(rng, 1, 1000), **kw)
            else:
                c = _append(min(seqs, 16), _log_int(rng, 17, 16384), past=rng.choice([0, 0, _log_int(rng, 1, 1000)]), **kw)
        else:
            longest = _log_int(rng, 1, 131072)
            c = _attention(seqs, longest if rng.random() < 0.3 else rng.randint(0, longest), longest, **kw)
    # no drawn case costs more than the largest listed one of its kind
    most = max((x for x in listed() if x["op"] == c["op"]), key=lambda x: work(x)["bytes"])
    while work(c)["bytes"] > work(most)["bytes"] or (c["op"] == "proj" and work(c)["flops"] > work(most)["flops"]):
        for k in {"norm": ["T"], "norm_bwd": ["T"], "append": ["tokens", "seqs"], "attention": ["longest", "shortest"], "proj": ["n_out"]}[c["op"]]:
            c[k] = c[k] * 3 // 4 | 1 if c[k] else 0
    # ... and the cache that an append case writes into stays small
    while c["op"] == "append" and sum(_lengths(c)) * c["kv_heads"] * c["head"] > 1 << 26:
        c["seqs"], c["past"] = max(1, c["seqs"] // 2), c["past"] // 2
    return c


def _lengths(case):
    """Lengths of the sequences, for an attention case shortest first, for an append case with the new tokens."""
    n = case["seqs"]
    if case["op"] == "append":
        # before them nothing, or about `past` tokens, an odd step apart
        return [new + (case["past"] + 7 * i if case["past"] else 0) for i, new in enumerate(_new_tokens(case))]
    lo, hi = case["shortest"], case["longest"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _new_tokens(case):
    """New tokens per sequence of an append case: one each, or uneven shares (1 : 2 : 3 ...) of all."""
    n, tokens = case["seqs"], case["tokens"]
    if not tokens:
        return [1] * n
    cuts = [tokens * i * (i + 1) // (n * (n + 1)) for i in range(n + 1)]
    return [b - a for a, b in zip(cuts, cuts[1:])]


_SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}


def work(case):
    op = case["op"]
    if op == "norm":
        n, e = case["T"] * case["d"], _SIZE[case["dtype"]]
        out = e if case["y"] == "same" else 1
        return {"bytes": n * (e + out + (2 * e if case["residual"] else 0)) + 4.0 * case["d"] + 8.0 * case["T"], "flops": 5.0 * n}
    if op == "norm_bwd":
        n, e = case["T"] * case["d"], _SIZE[case["dtype"]]
        return {"bytes": n * e * (4 if case["dsum"] else 3) + 8.0 * case["d"] + 4.0 * case["T"], "flops": 9.0 * n}
    if op == "proj":
        groups = case["n_out"] * (case["n_in"] // case["group"])
        return {"bytes": case["n_out"] * case["n_in"] / 2 + groups * (3.0 if case["zeros"] else 2.0) +
                case["T"] * (case["n_in"] * _SIZE[case["x"]] + case["n_out"] * _SIZE[case["y"]]),
                "flops": 2.0 * case["T"] * case["n_in"] * case["n_out"]}
    e = _SIZE[case["dtype"]]
    c = e if case["cache"] == "same" else 1
    row = case["kv_heads"] * (case["head"] * c + (0 if case["cache"] == "same" else 4))     # stored bytes of a token's keys
    if op == "append":
        t = sum(_new_tokens(case))
        return {"bytes": 2.0 * t * (case["kv_heads"] * case["head"] * e + row) + 8.0 * case["seqs"], "flops": 0.0}
    keys, q = sum(_lengths(case)), case["seqs"] * case["heads"]
    return {"bytes": 2.0 * keys * row + 2.0 * q * case["head"] * e + 4.0 * q + 4.0 * (keys // case["page"] + 2 * case["seqs"]),
            "flops": 4.0 * keys * case["heads"] * case["head"]}


class _State:
    pass


_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        # in slices: the caches are large, and what is drawn is fp32
        if len(shape) < 2 or math.prod(shape) < 1 << 26:
            return torch.randn(shape, generator=gen, device="cuda").to(dtype)
        out = torch.empty(shape, dtype=dtype, device="cuda")
        step = max(1, (1 << 26) // math.prod(shape[1:]))
        for i in range(0, shape[0], step):
            out[i:i + step] = torch.randn(out[i:i + step].shape, generator=gen, device="cuda").to(dtype)
        return out

    s = _State()
    s.case, op = case, case["op"]
    if op in ("norm", "norm_bwd"):
        T, d, dt = case["T"], case["d"], _TYPE[case["dtype"]]
        s.weight = 1.0 + 0.1 * normal(d)
        if op == "norm":
            s.x = normal(T, d, dtype=dt)
            s.residual = normal(T, d, dtype=dt) if case["residual"] else None
        else:
            # what the forward pass kept: the sum of the residual stream and its 1 / rms
            s.h = (1.4 * normal(T, d)).to(dt)
            s.rstd = (s.h.float().square().mean(1) + EPS).rsqrt()
            s.dy = normal(T, d, dtype=dt)
            s.dsum = normal(T, d, dtype=dt) if case["dsum"] else None
    elif op == "proj":
        T, n_in, n_out, groups = case["T"], case["n_in"], case["n_out"], case["n_in"] // case["group"]
        s.codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda", dtype=torch.uint8)
        s.scales = ((0.5 + torch.rand((n_out, groups), generator=gen, device="cuda")) * (0.02 / 4.6)).bfloat16()
        s.zeros = torch.randint(6, 10, (n_out, groups), generator=gen, device="cuda", dtype=torch.uint8) if case["zeros"] else None
        if case["x"] == "e4m3":
            x = normal(T, n_in)
            s.x_scale = x.abs().amax(1) / 448.0
            s.x = (x / s.x_scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            s.x, s.x_scale = normal(T, n_in, dtype=torch.bfloat16), None
    else:
        B, H, Hk, D, S = case["seqs"], case["heads"], case["kv_heads"], case["head"], case["page"]
        dt = _TYPE[case["dtype"]]
        order = torch.randperm(B, generator=gen, device="cuda")
        lens, T = torch.tensor(_lengths(case), device="cuda")[order], B
        s.seq_lens = lens.int()
        if op == "append":
            new, T = torch.tensor(_new_tokens(case), device="cuda")[order], sum(_new_tokens(case))
            s.offsets = torch.cat([new.new_zeros(1), new.cumsum(0)]).int() if case["tokens"] else None
        s.max_pages = max(1, -(-max(_lengths(case)) // S))
        # pages in the order that a program which hands them out and takes them back ends up with; -1: none
        need = (lens + S - 1) // S
        s.n_pages = sum(-(-n // S) for n in _lengths(case)) + 3
        pages = torch.randperm(s.n_pages, generator=gen, device="cuda").int()
        at = torch.arange(s.max_pages, device="cuda")
        first = torch.cat([need.new_zeros(1), need.cumsum(0)[:-1]])
        s.block_table = torch.where(at < need[:, None], pages[(first[:, None] + at).clamp(max=s.n_pages - 1)], -1).int().contiguous()
        if case["cache"] == "e4m3":
            stored = lambda: normal(s.n_pages, Hk, S, D, dtype=torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
            scale = lambda: 0.5 + torch.rand((s.n_pages, Hk, S), generator=gen, device="cuda")  # noqa: E731
            s.k_pages, s.v_pages, s.k_scale, s.v_scale = stored(), stored(), scale(), scale()
        else:
            s.k_pages, s.v_pages = normal(s.n_pages, Hk, S, D, dtype=dt), normal(s.n_pages, Hk, S, D, dtype=dt)
            s.k_scale = s.v_scale = None
        # rows as the projection leaves them: queries, keys and values of a token side by side
        qkv = normal(T, (H + 2 * Hk) * D, dtype=dt)
        s.q = qkv[:, :H * D].view(T, H, D)
        s.k = qkv[:, H * D:(H + Hk) * D].view(T, Hk, D)
        s.v = qkv[:, (H + Hk) * D:].view(T, Hk, D)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that calls the framework keeps: the call's configuration, output buffers, workspace."""
    import paper_2604_23108_amd as M
    c, op = s.case, s.case["op"]
    code = {"bf16": M.BF16, "f32": M.F32, "e4m3": M.E4M3}
    s.M = M
    if op in ("norm", "norm_bwd"):
        dt = _TYPE[c["dtype"]]
        like = dict(dtype=dt, device="cuda")
        if op == "norm":
            y8 = c["y"] == "e4m3"
            s.cfg = M.NormConfig(c["T"], c["d"], dtype=code[c["dtype"]], y_dtype=M.E4M3 if y8 else code[c["dtype"]], eps=EPS)
            s.sum_out = torch.empty((c["T"], c["d"]), **like) if c["residual"] else None
            s.y = torch.empty((c["T"], c["d"]), dtype=torch.uint8 if y8 else dt, device="cuda")
            s.y_scale = torch.empty(c["T"], device="cuda") if y8 else None
            s.rstd = torch.empty(c["T"], device="cuda")
        else:
            s.cfg = M.NormConfig(c["T"], c["d"], dtype=code[c["dtype"]], eps=EPS)
            s.dx, s.dweight = torch.empty((c["T"], c["d"]), **like), torch.empty(c["d"], device="cuda")
            s.workspace = torch.empty(max(16, M.mohge_norm_workspace_size(s.cfg)), dtype=torch.uint8, device="cuda")
    elif op == "proj":
        s.cfg = M.ProjConfig(c["T"], c["n_in"], c["n_out"], group=c["group"], x_dtype=code[c["x"]], y_dtype=code[c["y"]])
        s.y = torch.empty((c["T"], c["n_out"]), dtype=_TYPE[c["y"]], device="cuda")
    else:
        s.cfg = M.CacheConfig(c["seqs"], c["heads"], c["kv_heads"], c["head"], c["page"], s.n_pages, s.max_pages,
                              dtype=code[c["dtype"]], cache_dtype=code[c["dtype"] if c["cache"] == "same" else c["cache"]])
        if op == "attention":
            s.out = torch.empty((c["seqs"], c["heads"], c["head"]), dtype=_TYPE[c["dtype"]], device="cuda")
            s.lse = torch.empty((c["seqs"], c["heads"]), device="cuda")
            s.workspace = torch.zeros(max(16, M.mohge_cache_workspace_size(s.cfg)), dtype=torch.uint8, device="cuda")


def run(state):
    s = state
    op = s.case["op"]
    if own:
        return {"norm": _own_norm, "norm_bwd": _own_norm_bwd, "append": _own_append, "attention": _own_attention,
                "proj": _own_proj}[op](s)
    return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "append": _plain_append, "attention": _plain_attention,
            "proj": _plain_proj}[op](s)


# ---- the framework's calls ------------------------------------------------------------------------

def _values(codes):
    return codes.view(torch.float8_e4m3fn)


def _own_norm(s):
    s.M.mohge_rmsnorm(s.cfg, s.x, s.residual, s.weight, s.sum_out, s.y, s.y_scale, s.rstd)
    return {"sum": s.sum_out, "y": s.y if s.y_scale is None else _values(s.y), "y_scale": s.y_scale, "rstd": s.rstd}


def _own_norm_bwd(s):
    s.M.mohge_rmsnorm_bwd(s.cfg, s.dy, s.h, s.weight, s.rstd, s.dsum, s.dx, s.dweight, s.workspace)
    return {"dx": s.dx, "dweight": s.dweight}


def _own_append(s):
    s.M.mohge_cache_append(s.cfg, s.k, s.v, s.offsets, s.block_table, s.seq_lens, s.k_pages, s.v_pages, s.k_scale, s.v_scale)
    return _pages(s)


def _own_attention(s):
    s.M.mohge_cache_attention(s.cfg, s.q, s.block_table, s.seq_lens, s.k_pages, s.v_pages, s.k_scale, s.v_scale,
                              s.case["head"] ** -0.5, s.out, s.lse, s.workspace)
    return {"out": s.out, "lse": s.lse}


def _own_proj(s):
    s.M.mohge_proj_w4(s.cfg, s.x, s.x_scale, s.codes, s.scales, s.zeros, s.y)
    return {"y": s.y}


# ---- the plain forms ------------------------------------------------------------------------------

def _pages(s):
    if s.k_scale is None:
        return {"k_pages": s.k_pages, "v_pages": s.v_pages}
    return {"k_pages": _values(s.k_pages), "v_pages": _values(s.v_pages), "k_scale": s.k_scale, "v_scale": s.v_scale}


def _to_e4m3(y):
    """Codes and scales of the rows (last axis) of an fp32 tensor."""
    amax = y.abs().amax(-1)
    scale = torch.where(amax > 0, (amax / 448.0).clamp(min=2.0 ** -126), torch.ones_like(amax))
    return (y / scale.unsqueeze(-1)).to(torch.float8_e4m3fn), scale


def _plain_norm(s):
    dt = s.x.dtype
    h = s.x.float() if s.residual is None else s.x.float() + s.residual.float()
    rstd = (h.square().mean(1) + EPS).rsqrt()
    y = h * rstd[:, None] * s.weight
    out = {"sum": None if s.residual is None else h.to(dt), "y": None, "y_scale": None, "rstd": rstd}
    if s.case["y"] == "e4m3":
        out["y"], out["y_scale"] = _to_e4m3(y)
    else:
        out["y"] = y.to(dt)
    return out


def _plain_norm_bwd(s):
    n = s.h.float() * s.rstd[:, None]
    dy = s.dy.float()
    g = s.weight * dy
    dx = s.rstd[:, None] * (g - n * (g * n).mean(1, keepdim=True))
    if s.dsum is not None:
        dx = dx + s.dsum.float()
    return {"dx": dx.to(s.h.dtype), "dweight": (dy * n).sum(0)}


def _plain_append(s):
    B, S = s.case["seqs"], s.case["page"]
    if s.offsets is None:
        seq, pos = torch.arange(B, device="cuda"), s.seq_lens.long() - 1
    else:
        off = s.offsets.long()
        t = torch.arange(s.k.shape[0], device="cuda")
        seq = torch.searchsorted(off[1:], t, right=True)
        pos = s.seq_lens.long()[seq] - off[seq + 1] + t
    page, slot = s.block_table[seq, pos // S].long(), pos % S
    if s.k_scale is None:
        s.k_pages[page, :, slot] = s.k
        s.v_pages[page, :, slot] = s.v
    else:
        for rows, pages, scales in ((s.k, s.k_pages, s.k_scale), (s.v, s.v_pages, s.v_scale)):
            codes, scale = _to_e4m3(rows.float())
            pages[page, :, slot] = codes.view(torch.uint8)
            scales[page, :, slot] = scale
    return _pages(s)


def _gathered(s, pages, scales):
    """[seqs, kv heads, positions, head] in fp32."""
    c = s.case
    at = s.block_table.long().clamp(min=0)
    x = (pages if scales is None else _values(pages))[at].float()
    if scales is not None:
        x = x * scales[at].unsqueeze(-1)
    return x.permute(0, 2, 1, 3, 4).reshape(c["seqs"], c["kv_heads"], s.max_pages * c["page"], c["head"])


def _plain_attention(s):
    c = s.case
    B, Hk, G, D = c["seqs"], c["kv_heads"], c["heads"] // c["kv_heads"], c["head"]
    q = s.q.float().reshape(B, Hk, G, D)
    z = torch.matmul(q, _gathered(s, s.k_pages, s.k_scale).transpose(2, 3)) * D ** -0.5
    there = torch.arange(z.shape[3], device="cuda") < s.seq_lens[:, None]
    z = torch.where(there[:, None, None], z, -math.inf)
    top = z.amax(3, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(3, keepdim=True)
    v = torch.where(there[:, None, :, None], _gathered(s, s.v_pages, s.v_scale), 0.0)
    out = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = top.squeeze(3) + torch.log(total.squeeze(3))
    return {"out": out.reshape(B, Hk * G, D).to(s.q.dtype), "lse": lse.reshape(B, Hk * G)}


def _plain_proj(s):
    c = s.case
    groups = c["n_in"] // c["group"]
    codes = torch.stack([s.codes & 15, s.codes >> 4], dim=2).reshape(c["n_out"], groups, c["group"])
    zeros = 8.0 if s.zeros is None else s.zeros.float().unsqueeze(2)
    w = ((codes.float() - zeros) * s.scales.float().unsqueeze(2)).reshape(c["n_out"], c["n_in"])
    x = s.x.float() if s.x_scale is None else _values(s.x).float() * s.x_scale[:, None]
    return {"y": torch.matmul(x, w.T).to(_TYPE[c["y"]])}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = s.x.double()
        if s.residual is not None:
            h = h + s.residual.double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / case["d"] + EPS)
        y = s.weight.double() * (rstd[:, None] * h)
        out = {"sum": None if s.residual is None else h, "y": y, "y_scale": None, "rstd": rstd}
        if case["y"] == "e4m3":
            # the values before they are rounded to codes
            out["y_scale"] = y.abs().max(1).values / 448.0
            out["y"] = y / out["y_scale"][:, None]
        return out
    if op == "norm_bwd":
        h, dy, r, w = s.h.double(), s.dy.double(), s.rstd.double()[:, None], s.weight.double()
        inner = (dy * w * h).sum(1, keepdim=True)
        dx = r * w * dy - h * inner * r ** 3 / case["d"]
        if s.dsum is not None:
            dx = dx + s.dsum.double()
        return {"dx": dx, "dweight": torch.einsum("td,td->d", dy, h * r)}
    if op == "append":
        new, S = _new_tokens(case), case["page"]
        out = {}
        rows_of = []                                           # (page, offset) of every row of k and v
        table, lens = s.block_table.cpu(), s.seq_lens.cpu().tolist()
        counts = [1] * case["seqs"] if s.offsets is None else s.offsets.diff().cpu().tolist()
        assert sorted(counts) == sorted(new)
        for b, n in enumerate(counts):
            rows_of += [(int(table[b, p // S]), p % S) for p in range(lens[b] - n, lens[b])]
        page = torch.tensor([p for p, _ in rows_of], device="cuda")
        slot = torch.tensor([o for _, o in rows_of], device="cuda")
        for name, rows, pages, scales in (("k", s.k, s.k_pages, s.k_scale), ("v", s.v, s.v_pages, s.v_scale)):
            if scales is None:
                x = pages.double()
                x[page, :, slot] = rows.double()
            else:
                x, sc, r = _values(pages).double(), scales.double(), rows.double()
                top = r.abs().max(2).values / 448.0
                x[page, :, slot] = r / top[:, :, None]
                sc[page, :, slot] = top
                out[name + "_scale"] = sc
            out[name + "_pages"] = x
        return out
    if op == "attention":
        Hk, G, D, S = case["kv_heads"], case["heads"] // case["kv_heads"], case["head"], case["page"]
        out = torch.zeros((case["seqs"], case["heads"], D), dtype=torch.float64, device="cuda")
        lse = torch.full((case["seqs"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(s.seq_lens.cpu().tolist()):
            if n == 0:
                continue
            pages = s.block_table[b, :-(-n // S)].long()
            kv = []
            for store, scales in ((s.k_pages, s.k_scale), (s.v_pages, s.v_scale)):
                x = store[pages].double() if scales is None else _values(store[pages]).double() * scales[pages].double()[..., None]
                kv.append(x.transpose(0, 1).reshape(Hk, -1, D)[:, :n])
            z = s.q[b].double().view(Hk, G, D) @ kv[0].transpose(1, 2) / math.sqrt(D)
            lse[b] = torch.logsumexp(z, 2).reshape(-1)
            out[b] = (torch.softmax(z, 2) @ kv[1]).reshape(-1, D)
        return {"out": out, "lse": lse}
    groups, n_out = case["n_in"] // case["group"], case["n_out"]
    x = (s.x.double() if s.x_scale is None else _values(s.x).double() * s.x_scale.double()[:, None]).view(case["T"], groups, -1)
    y = torch.empty((case["T"], n_out), dtype=torch.float64, device="cuda")
    for i in range(0, n_out, 4096):
        part = s.codes[i:i + 4096]
        w = torch.empty((part.shape[0], case["n_in"]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (part % 16).double(), (part // 16).double()
        w = w.view(-1, groups, case["group"])
        w = (w - (8.0 if s.zeros is None else s.zeros[i:i + 4096].double()[:, :, None])) * s.scales[i:i + 4096].double()[:, :, None]
        y[:, i:i + 4096] = x.reshape(case["T"], -1) @ w.reshape(-1, case["n_in"]).T
    return {"y": y}
