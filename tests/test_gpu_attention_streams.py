"""Calls of attention that run at the same time: graphs on several streams, plain calls beside them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()


def test_graphs_of_one_cache_run_at_the_same_time():
    """Two graphs captured one after the other on the stream that torch captures on, replayed on two streams, beside plain calls on a third: each gives what it gives alone.
    (The sequence lies in many waves' shares, whose sums go through the workspace.)"""
    from paper_2404_01847_amd.attention import PagedKV
    n, page, hq, hkv, d = 20000, 64, 32, 8, 128
    cache = PagedKV(-(-n // page), page, hkv, d)
    at = torch.arange(n, device="cuda")
    cache.write(normal((n, hkv, d), 1), normal((n, hkv, d), 2), at)
    table = torch.arange(cache.pages, dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    Q = [normal((1, hq, d), 3 + i) for i in range(3)]
    want = [cache.attend(q, table, lengths, torch.empty_like(q)).clone() for q in Q]
    O = [torch.empty_like(q) for q in Q]
    graphs = []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(Q[i], table, lengths, O[i])
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(10):
        for o in O:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(5):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
            with torch.cuda.stream(streams[2]):
                cache.attend(Q[2], table, lengths, O[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(O, want))
