"""Layers that share a page table and lengths, cut down together: each keeps the tokens that its own weights name."""
import numpy as np
import pytest
import torch

from tests.test_gpu_evict import keep_reference, weights
from tests.test_gpu_new_tokens import i32, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("four_bits", [False, True])
@pytest.mark.parametrize("captured", [False, True])
def test_layers_that_share_their_lengths(four_bits, captured):
    import paper_2502_02770_amd as T
    B, hq, hkv, pages, lens = 2, 8, 2, 9, [130, 77]
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    seq = i32(lens)
    make = T.PagedKV4 if four_bits else T.PagedKV
    layers = [make(hq, hkv, table, seq, B * pages) for _ in range(3)]
    assert all(c.seq_lens.data_ptr() == seq.data_ptr() for c in layers)
    budget, m = [40, 50], [T.TokenMass(c) for c in layers]
    k, v = (torch.empty(144 * B, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pools = ("kq_pool", "kq_meta", "vq_pool", "vq_meta") if four_bits else ("k_pool", "v_pool", "kq_pool", "kq_meta")

    def begin():
        """-> every layer's rows in order of position, and its weights"""
        seq.copy_(i32(lens))
        was = []
        for i, (c, x) in enumerate(zip(layers, m)):
            k.copy_(queries(144 * B, hkv, 2 * i))
            v.copy_(queries(144 * B, hkv, 2 * i + 1))
            c.append(k, v, i32([0, 0]), i32(lens), i32([0, 144]), 144)
            x.mass.copy_(torch.from_numpy(weights(B, pages * 16, i)))
            was.append([rows(c, p) for p in pools])
        return was

    def rows(c, pool):
        return getattr(c, pool)[table.long()].transpose(2, 3).reshape(B, pages * 16, hkv, -1).clone()

    cut = lambda: m[0].evict(i32(budget) if not captured else held, 2, 8, others=m[1:])  # noqa: E731
    held = i32(budget)
    if captured:
        begin()
        cut()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cut()
        cut = graph.replay
    for _ in range(2):
        was = begin()
        cut()
        torch.cuda.synchronize()
        assert seq.tolist() == budget
        for i, (c, x) in enumerate(zip(layers, m)):
            w = weights(B, pages * 16, i)
            for b in range(B):
                want = keep_reference(w[b], lens[b], budget[b], 2, 8, 10**6)
                assert np.array_equal(x.keep_idx[b, :budget[b]].cpu().numpy(), want), (i, b)
                assert np.array_equal(x.mass[b, :budget[b]].cpu().numpy(), w[b][want]) and (x.mass[b, budget[b]:] == 0).all()
                for j, p in enumerate(pools):
                    assert torch.equal(rows(c, p)[b, :budget[b]].view(torch.uint8), was[i][j][b, torch.from_numpy(want).long().cuda()].view(torch.uint8)), (i, b, p)


def test_layers_of_another_batch_are_refused():
    import paper_2502_02770_amd as T
    table = torch.arange(4, dtype=torch.int32).view(2, 2)
    two = T.TokenMass(T.PagedKV4(8, 2, table, torch.tensor([20, 20], dtype=torch.int32), 4))
    one = T.TokenMass(T.PagedKV4(8, 2, table[:1], torch.tensor([20], dtype=torch.int32), 4))
    with pytest.raises(AssertionError, match="one batch"):
        two.evict(i32([5, 5]), others=[one])
    assert two.cache.seq_lens.tolist() == [20, 20]
