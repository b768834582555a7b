"""Rotation, appending and chunks at the same time as other calls, on other streams, and within larger buffers: nothing is written but what is theirs."""
import math

import pytest
import torch

from test_gpu_attention_guards import Guarded, i32, normal, offsets
from test_gpu_rotary import Case, empty_cache, scattered

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("gap", [0, 8])
@pytest.mark.parametrize("norms", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("tokens,hq,hkv,d,rotated", [(1, 1, 1, 16, 16), (33, 6, 2, 80, 80), (700, 17, 3, 64, 32), (5, 9, 9, 128, 0), (2100, 8, 1, 112, 112)])
def test_rotation_stays_in_its_operands(tokens, hq, hkv, d, rotated, norms, gap):
    import paper_2404_01847_amd as s24
    c, new = Case(tokens, hq, hkv, d, BF16, rotated, norms), Guarded()
    Q, K = new((tokens, hq, d), BF16, gap), new((tokens, hkv, d), BF16, gap)
    s24.rotary_fwd(c.layer.plan, c.Q, c.K, c.positions, Q, K)
    new.check("forward")
    dQ, dK, dwq, dwk = new((tokens, hq, d), BF16, gap), new((tokens, hkv, d), BF16, gap), new((d,), torch.float32), new((d,), torch.float32)
    work = new((s24.rotary_bwd_workspace(c.layer.plan, tokens, hq, hkv),), torch.uint8)
    s24.rotary_bwd(c.layer.plan, c.dQ, c.dK, c.Q, c.K, c.positions, dQ, dK, dwq, dwk, 0.0, work if work.numel() else None)
    new.check("backward")
    want = c.layer.forward(c.Q, c.K, c.positions)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and all(x.isfinite().all() for x in (dQ, dK))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tokens,hq,hkv,d,page", [(1, 4, 1, 64, 16), (50, 6, 3, 80, 32), (1600, 8, 8, 128, 64), (1900, 6, 6, 48, 16)])
def test_appending_stays_in_its_operands(tokens, hq, hkv, d, page, bits):
    """With places that are the cache's, and with places that hold anything."""
    import paper_2404_01847_amd as s24
    c, new = Case(tokens, hq, hkv, d, BF16), Guarded()
    places, pages = scattered(tokens, page, tokens)
    held = [new((pages, hkv, page, d), torch.uint8 if bits == 8 else BF16) for _ in range(2)]
    steps = [new((pages, hkv, page), torch.float32) for _ in range(2)] if bits == 8 else []
    cache = s24.KVBuffers(*held, BF16, *steps)
    Q = new((tokens, hq, d), BF16, 8)
    s24.kv_append(cache, c.layer.plan, c.Q, c.K, c.V, c.positions, places, Q)
    new.check("appended")
    gen = torch.Generator().manual_seed(4)
    s24.kv_append(cache, c.layer.plan, c.Q, c.K, c.V, c.positions, torch.randint(-(1 << 40), 1 << 40, (tokens,), generator=gen).cuda(), Q)
    s24.kv_append(cache, c.layer.plan, c.Q, c.K, c.V, c.positions, torch.arange(tokens, device="cuda") + pages * page - tokens // 2, Q)
    new.check("anything")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lens,new_tokens,hq,hkv,d,page", [([9000, 1, 300], [50, 1, 7], 8, 2, 128, 64), ([0, 70, 128], [0, 70, 3], 12, 12, 64, 16), ([500] * 70, [3] * 70, 4, 1, 80, 32),
                                                           ([2000, 3000], [900, 30], 16, 2, 112, 16), ([5000], [1], 32, 1, 64, 128)])
def test_chunks_stay_in_their_operands(lens, new_tokens, hq, hkv, d, page, bits):
    """Whole tiles, and pieces of them with their sums in the workspace."""
    import paper_2404_01847_amd as s24
    counts = [-(-x // page) for x in lens]
    pages, n = sum(counts), sum(lens)
    table, places, at = torch.zeros((len(lens), max(counts)), dtype=torch.int32), [], 0
    for i, (x, k) in enumerate(zip(lens, counts)):
        table[i, :k] = torch.arange(at, at + k)
        places.append(torch.arange(x) + at * page)
        at += k
    cache = empty_cache(pages, page, hkv, d, BF16, bits)
    cache.write(normal((n, hkv, d), BF16, 1), normal((n, hkv, d), BF16, 2), torch.cat(places).cuda())
    tokens, new = sum(new_tokens), Guarded()
    Q, O = normal((tokens, hq, d), BF16, 3), new((tokens, hq, d), BF16, 8)
    work = new((s24.attn_chunk_workspace(cache.buffers, table.shape[1], tokens, len(lens), hq),), torch.uint8)
    s24.attn_chunk(cache.buffers, Q, i32(offsets(new_tokens)), table.cuda(), i32(lens), O, work if work.numel() else None)
    new.check("attended")
    want = cache.attend_chunk(Q, i32(offsets(new_tokens)), table.cuda(), i32(lens), torch.empty_like(Q))
    assert O.isfinite().all() and torch.equal(O, want)


def test_graphs_of_one_layer_and_cache_run_at_the_same_time():
    """Two graphs of chunks, and one of gradients, captured one after the other and replayed on streams of their own beside plain calls: each gives what it gives alone.  (All of
    them have sums in a workspace.)"""
    from paper_2404_01847_amd.attention import PagedKV
    n, page, hq, hkv, d = 6000, 64, 8, 2, 128
    cache = PagedKV(-(-n // page), page, hkv, d)
    at = torch.arange(n, device="cuda")
    cache.write(normal((n, hkv, d), BF16, 1), normal((n, hkv, d), BF16, 2), at)
    table, lengths, cu = torch.arange(cache.pages, dtype=torch.int32, device="cuda")[None], i32([n]), i32([0, 40])
    Q = [normal((40, hq, d), BF16, 3 + i) for i in range(3)]
    want = [cache.attend_chunk(q, cu, table, lengths, torch.empty_like(q)).clone() for q in Q]
    c = Case(900, hq, hkv, d, BF16)
    grads = tuple(torch.empty_like(x) for x in (c.dQ, c.dK))
    backward = lambda: c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=grads)
    backward()
    want_w = c.layer.dwq.clone(), c.layer.dwk.clone()
    O = [torch.empty_like(q) for q in Q]
    graphs = []
    for call in (lambda: cache.attend_chunk(Q[0], cu, table, lengths, O[0]), lambda: cache.attend_chunk(Q[1], cu, table, lengths, O[1]), backward):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(6):
        for x in (*O, c.layer.dwq, c.layer.dwk):
            x.fill_(math.nan)
        torch.cuda.synchronize()
        for _ in range(4):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
            with torch.cuda.stream(streams[3]):
                cache.attend_chunk(Q[2], cu, table, lengths, O[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(O, want))
        assert torch.equal(c.layer.dwq, want_w[0]) and torch.equal(c.layer.dwk, want_w[1])


def test_appended_then_attended_on_one_stream():
    """The calls as they follow each other in serving, on another stream than the default one, captured as a whole and replayed: new tokens appended, and attended over."""
    tokens, hq, hkv, d, page = 48, 8, 2, 64, 16
    c = Case(tokens, hq, hkv, d, BF16, seed=7)
    cache = empty_cache(12, page, hkv, d, BF16, 8)
    table = torch.tensor([[3, 1, 7, 0], [2, 5, 9, 4]], dtype=torch.int32, device="cuda")
    rows = torch.cat([torch.arange(30), torch.arange(18)]).cuda()
    sequence = torch.tensor([0] * 30 + [1] * 18, device="cuda")
    places = table[sequence, rows // page].long() * page + rows % page
    cu, lengths, O = i32([0, 30, 48]), i32([30, 18]), torch.empty((tokens, hq, d), dtype=BF16, device="cuda")

    def serve():
        Q = cache.append(c.layer, c.Q, c.K, c.V, c.positions, places)
        return cache.attend_chunk(Q, cu, table, lengths, O)

    want = serve().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in (cache.K, cache.V, cache.k_step, cache.v_step, O):
            x.zero_()
        serve()
    side.synchronize()
    assert torch.equal(O, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        serve()
    for _ in range(3):
        for x in (cache.K, cache.V, cache.k_step, cache.v_step, O):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


def test_plans_of_another_device_and_offsets_past_32_bits():
    """Heads that lie 2^31 values apart, as operands and as results."""
    import paper_2404_01847_amd as s24
    n, d, gap = 70, 64, 1 << 31
    c = Case(n, 2, 2, d, BF16, views="whole")
    want = [x.clone() for x in c.layer.forward(c.Q, c.K, c.positions)]
    flat = torch.empty(gap + n * d, dtype=BF16, device="cuda")
    apart = flat.as_strided((n, 2, d), (d, gap, 1))
    apart.copy_(c.Q)
    s24.rotary_fwd(c.layer.plan, apart, c.K, c.positions, c.layer.Q, c.layer.K)
    assert torch.equal(c.layer.Q, want[0])
    s24.rotary_fwd(c.layer.plan, c.Q, c.K, c.positions, apart, c.layer.K)
    assert torch.equal(apart, want[0])
    with pytest.raises(ValueError, match="the plan lies on"):
        s24.rotary_fwd(c.layer.plan, c.Q.cpu(), c.K.cpu(), c.positions.cpu(), c.Q.cpu(), c.K.cpu())
