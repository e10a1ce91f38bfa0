"""Counters of the attention's workspace that were not zero: results that are joined from parts are NaN in that call and in the next, whatever
small number a counter held (as many as there are parts, one less, a negative one), and right again once the workspace is cleared."""
import pytest
import torch

import paper_2604_23108_amd as M
from test_gpu_cache import _check, _filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[9000, 40], [700, 40]])
def test_no_residue_is_taken_for_parts(lens):
    """Rows of dozens of parts and of three or so; the second sequence is not cut and stays right."""
    cfg = M.CacheConfig(2, 8, 2, 128, 16, 800, 600)
    q, table, n, kp, vp, ks, vs = _filled(cfg, lens, 6)
    out, lse = torch.empty_like(q).contiguous(), torch.empty((2, 8), device="cuda")
    ws = torch.zeros(M.mohge_cache_workspace_size(cfg), dtype=torch.uint8, device="cuda")

    def attend():
        out.fill_(7.0)
        lse.fill_(7.0)
        M.mohge_cache_attention(cfg, q, table, n, kp, vp, ks, vs, 128 ** -0.5, out, lse, ws)

    attend()
    _check(cfg, q, table, n, kp, vp, ks, vs, 128 ** -0.5, out, lse)
    good, good_lse = out.clone(), lse.clone()
    words = {torch.int64: 4, torch.int32: 8, torch.uint8: 32}               # the counters of both rows of both sequences
    for residue in [*range(1, 90), 255, -1, -2, -36]:
        for kind, count in words.items():
            if not torch.iinfo(kind).min <= residue <= torch.iinfo(kind).max:
                continue
            ws.zero_()
            ws.view(kind)[:count] = residue
            for call in range(3):
                attend()
                assert out[0].isnan().all() and lse[0].isnan().all(), (residue, kind, call)
                assert torch.equal(out[1], good[1]) and torch.equal(lse[1], good_lse[1]), (residue, kind, call)
    ws.zero_()
    attend()
    assert torch.equal(out, good) and torch.equal(lse, good_lse) and (ws[:32] == 0).all()
