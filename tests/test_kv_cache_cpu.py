"""Which rows an append writes after sequences have grown unevenly (host side of KVCache)."""
import pytest
import torch

import paper_2604_23108_amd as M
from paper_2604_23108_amd import block_binding as B


@pytest.fixture
def appended(monkeypatch):
    """The lengths and offsets that every append hands on; a length of 0 leaves a sequence's row out."""
    calls = []
    monkeypatch.setattr(B, "mohge_cache_append", lambda cfg, k, v, offsets, table, lens, *rest: calls.append((lens.tolist(), offsets)))
    return calls


def test_a_row_goes_only_to_sequences_that_grew(appended):
    kv = M.KVCache(M.CacheConfig(n_seqs=5, n_heads=4, n_kv_heads=2, head_size=64, page_size=16, n_pages=30, max_pages=6), device="cpu")
    kv.append(None, None)
    assert appended.pop()[0] == [0, 0, 0, 0, 0]
    steps = [([3, 0, 17, 1, 0], [3, 0, 17, 1, 0], [3, 0, 17, 1, 0]),
             ([1, 0, 1, 0, 0], [4, 0, 18, 1, 0], [4, 0, 18, 0, 0]),          # the fourth keeps its last position
             ([0, 0, 0, 0, 0], [4, 0, 18, 1, 0], [0, 0, 0, 0, 0]),
             ([1, 1, 1, 1, 1], [5, 1, 19, 2, 1], [5, 1, 19, 2, 1]),
             ([1, 1, 1, 1, 1], [6, 2, 20, 3, 2], [6, 2, 20, 3, 2]),
             ([0, 2, 1, 30, 1], [6, 4, 21, 33, 3], [0, 4, 21, 33, 3]),
             ([2, 2, 2, 2, 2], [8, 6, 23, 35, 5], [8, 6, 23, 35, 5])]
    lens = kv.seq_lens
    for new, lengths, want in steps:
        kv.grow(new)
        assert kv.lengths == lengths and kv.seq_lens.tolist() == lengths
        for _ in range(2):
            kv.append(None, None)
            assert appended.pop()[0] == want, new
    offsets = torch.tensor([0, 1, 1, 1, 1, 1], dtype=torch.int32)
    kv.append(None, None, offsets)                                           # offsets say for themselves which rows there are
    assert appended.pop() == (lengths, offsets)
    kv.free(2)
    kv.free(-1)
    kv.append(None, None)
    assert appended.pop()[0] == [8, 6, 0, 35, 0] and kv.seq_lens.tolist() == [8, 6, 0, 35, 0]
    kv.grow([1, 1, 0, 1, 0])
    kv.append(None, None)
    assert appended.pop()[0] == [9, 7, 0, 36, 0] == kv.lengths
    assert kv.seq_lens is lens                                               # (a recorded step reads the same tensors)


@pytest.mark.gpu
def test_a_sequence_that_did_not_grow_keeps_its_rows_also_in_a_graph():
    kv = M.KVCache(M.CacheConfig(n_seqs=3, n_heads=4, n_kv_heads=2, head_size=64, page_size=16, n_pages=12, max_pages=4))
    k, v = (torch.randn((3, 2, 64), device="cuda").bfloat16() for _ in range(2))
    kv.grow([1, 1, 1])
    kv.append(k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.append(k, v)
    rows = lambda b, n: (kv.k_pages[kv.pages[b][0], :, n].clone(), kv.v_pages[kv.pages[b][0], :, n].clone())  # noqa: E731
    for i, new in enumerate(([1, 0, 1], [0, 1, 1], [1, 1, 1], [0, 0, 1])):
        last = [rows(b, n - 1) for b, n in enumerate(kv.lengths)]
        k.add_(1)
        v.sub_(1)
        kv.grow(new)
        (graph.replay if i % 2 else lambda: kv.append(k, v))()
        for b, n in enumerate(kv.lengths):
            want = (k[b], v[b]) if new[b] else last[b]
            assert all(torch.equal(a, w) for a, w in zip(rows(b, n - 1), want)), (new, b)
            if new[b] and n > 1:
                assert all(torch.equal(a, w) for a, w in zip(rows(b, n - 2), last[b])), (new, b)
