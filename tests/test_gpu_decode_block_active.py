"""Sequences that sit steps of a decoder block out: paused ones keep their cache, freed ones take no pages, one at the end of its block
table does not stop the others."""
import pytest
import torch

import paper_2604_23108_amd as M
from paper_2604_23108_amd.decode_block import random_block

pytestmark = pytest.mark.gpu


def test_sequences_that_sit_steps_out():
    part, whole = (random_block(4, page_size=16, longest=32, seed=2) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda: torch.randn((4, 1024), generator=gen, device="cuda").bfloat16()  # noqa: E731
    for _ in range(20):                                                # the second page of two
        x = draw()
        part.forward(x)
        whole.forward(x)
    cache = part.cache
    rows = lambda b: [p[torch.tensor(cache.pages[b], device="cuda")].clone() for p in (cache.k_pages, cache.v_pages)]  # noqa: E731
    kept = rows(1)
    cache.free(2)
    for step in range(12):                                             # sequences 0 and 3 go on, 1 pauses, 2 is finished
        x = draw()
        part.forward(x, active=[True, False, False, True])
        whole.forward(x)
        # a short sequence's attention is one workgroup's: the same bits whatever the others do
        assert torch.equal(cache.out[[0, 3]], whole.cache.out[[0, 3]]) and (cache.out[2] == 0).all(), step
        y, want = part.layer.y[[0, 3]].double(), whole.layer.y[[0, 3]].double()
        assert y.isfinite().all() and (y - want).abs().max() <= 2.0 ** -6 * want.abs().max(), step
    assert cache.lengths == [32, 20, 0, 32] == cache.seq_lens.tolist()
    assert all(torch.equal(a, b) for a, b in zip(rows(1), kept)) and cache.pages[2] == []
    # 0 and 3 are at the end of the table: all together has no room, the others go on
    with pytest.raises(M.MohgeError, match="max_pages|pages needed"):
        part.forward(draw())
    part.forward(draw(), active=[0, 1, 1, 0])
    assert cache.lengths == [32, 21, 1, 32] == cache.seq_lens.tolist()
    with pytest.raises(M.MohgeError, match="count for each"):
        part.forward(draw(), active=[True])
