"""The operators around the layer together: steps of a decoder block against the definitions in 64 bits, stage by stage, and a training
step of the norm in front of the layer."""
import numpy as np
import pytest
import torch

import paper_2604_23108_amd as M
from paper_2604_23108_amd.decode_block import main, random_block

pytestmark = pytest.mark.gpu


def _near(got, want, rel):
    """Rounding of a bf16 result, and `rel` of the tensor's size for what enters with it."""
    got, want = got.double(), want.double()
    assert got.isfinite().all()
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + rel * want.abs().max()).all(), float((got - want).abs().max() / want.abs().max())


def _norm(s, w, eps=1e-6):
    return s / torch.sqrt(s.square().mean(1, keepdim=True) + eps) * w.double()


def _weights(p):
    c = torch.stack([p.codes & 15, p.codes >> 4], 2).reshape(p.cfg.n_out, -1, p.cfg.group).double()
    return ((c - 8) * p.scales.double()[:, :, None]).reshape(p.cfg.n_out, -1)


@pytest.mark.parametrize("seqs,cache,norm_8bit", [(1, M.BF16, True), (7, M.BF16, False), (32, M.E4M3, True)])
def test_steps_of_a_block(seqs, cache, norm_8bit):
    block = random_block(seqs, page_size=16, longest=64, cache_dtype=cache, norm_8bit=norm_8bit, seed=seqs)
    c = block.cache.cfg
    gen = torch.Generator(device="cuda").manual_seed(7)
    residual, keys, values = None, [], []
    for step in range(20):                                  # over a page's end
        x = torch.randn((seqs, 1024), generator=gen, device="cuda").bfloat16()
        y, stream = block.forward(x, residual)
        torch.cuda.synchronize()
        s = x.double() + (0 if residual is None else residual.double())
        h = _norm(s, block.attention_norm.weight)
        if norm_8bit:
            got = block.attention_norm.y.view(torch.float8_e4m3fn).double() * block.attention_norm.y_scale.double()[:, None]
            assert ((got - h).abs() <= 2.0 ** -4 * h.abs() + 2.0 ** -9 * block.attention_norm.y_scale.double()[:, None]).all()
        else:
            got = block.attention_norm.y.double()
            _near(got, h, 1e-6)
        # every stage from what the stage before handed on
        qkv = got @ _weights(block.qkv).T.contiguous()
        _near(block.qkv.y, qkv, 1e-5)
        q, k, v = block.qkv.y.double().split([1024, 256, 256], 1)
        for rows, kept in ((k, keys), (v, values)):
            rows = rows.reshape(seqs, 4, 64)
            if cache == M.E4M3:
                scale = rows.abs().amax(2, keepdim=True) / 448
                rows = (rows / scale).float().to(torch.float8_e4m3fn).double() * scale
            kept.append(rows)
        kk, vv = torch.stack(keys, 2), torch.stack(values, 2)                # [seqs, kv heads, positions, size]
        z = q.reshape(seqs, 4, 4, 64) @ kk.transpose(2, 3).contiguous() / 8
        out = (torch.softmax(z, 3) @ vv).reshape(seqs, 16, 64)
        # E4M3: a key that lies between two codes may have got the other one (fp32 scale): 2^-4 of an element, here and there
        _near(block.cache.out, out, 2e-2 if cache == M.E4M3 else 1e-4)
        a = block.cache.out.double().reshape(seqs, 1024) @ _weights(block.out).T.contiguous()
        _near(block.out.y, a, 1e-5)
        _near(stream, block.out.y.double() + s.float().bfloat16().double(), 1e-6)
        _near(block.layer_norm.y, _norm(block.out.y.double() + s.float().bfloat16().double(), block.layer_norm.weight), 1e-6)
        assert torch.equal(y, block.layer.forward(block.layer_norm.y))
        residual = stream.clone()
    assert block.cache.lengths == [20] * seqs and block.cache.seq_lens.tolist() == [20] * seqs


def test_a_step_in_a_graph():
    block = random_block(5, page_size=16, longest=128, seed=3)
    x = torch.randn((5, 1024), device="cuda").bfloat16()
    residual = torch.randn((5, 1024), device="cuda").bfloat16()
    block.forward(x, residual)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.step(x, residual)
    for i in range(20):
        block.cache.grow([1] * 5)
        x.copy_(torch.randn((5, 1024), device="cuda"))
        y, stream = (t.clone() for t in block.step(x, residual))
        torch.cuda.synchronize()
        block.layer.y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(block.layer.y, y) and torch.equal(block.layer_norm.sum, stream), i


def test_the_command(capsys):
    main(["--seqs", "4", "--steps", "3", "--prompt", "70", "--cache-8bit"])
    assert "4 sequences of 76 positions" in capsys.readouterr().out


def test_a_training_step_of_the_norm_in_front_of_the_layer():
    """Gradient through norm and layer: the layer's dx is the norm's dy, dy past the layer reaches the residual stream."""
    from gpu_harness import DeviceLayer, to_dev
    from synth import Workload, generate
    w = Workload("normed", T=333, d=256, n_groups=3, experts_per_group=4, d_ff=(64, 128, 192), k_groups=2, k_experts=4, seed=5,
                 training=True)
    inp = generate(w)
    dl = DeviceLayer(w, inp, backward=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    residual = torch.randn((333, 256), generator=gen, device="cuda").bfloat16()
    weight = 1 + 0.1 * torch.randn(256, generator=gen, device="cuda")
    norm = M.ResidualNorm(M.NormConfig(333, 256), weight, backward=True)
    h = norm.forward(dl.x, residual)
    dl.layer.forward(h)
    dy = to_dev(inp.dy, True)
    dh = dl.layer.backward(h, dy)
    dx = norm.backward(dh, dy)
    torch.cuda.synchronize()
    s, r = norm.sum.double(), norm.rstd.double()[:, None]
    g, n = weight.double() * dh.double(), s * r
    want = dy.double() + r * (g - n * (g * n).mean(1, keepdim=True))
    _near(dx, want, 1e-5)
    dw = (dh.double() * n).sum(0)
    assert ((norm.dweight.double() - dw).abs() <= 400 * 2.0 ** -24 * (dh.double() * n).abs().sum(0)).all()
    assert np.isfinite(dl.layer.dw_group.cpu().numpy()).all()
