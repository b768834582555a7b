"""Attention on the GPU against 64 bits on the CPU (attention_reference.py, which derives the bounds)."""
import math
import random

import pytest
import torch

from attention_reference import OPERAND_TINY, TINY, U, assert_within, packed, quantise

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def s24():
    import paper_2404_01847_amd as s24
    return s24


def offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def gpu_i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def normal(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def run(s24, lq, lk, hq, hkv, d, dtype, causal=True, scale=None, views="projection", seed=0, backward=True, qstd=1.0):
    cq, ck = offsets(lq), offsets(lk)
    tq, tk = cq[-1], ck[-1]
    if views == "projection" and lq == lk:
        x = normal((tq, hq + 2 * hkv, d), dtype, seed)
        x[:, :hq] *= qstd
        Q, K, V = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    elif views == "heads":      # [heads][tokens][d] buffers
        Q, K, V = (normal((h, t, d), dtype, seed + i).transpose(0, 1) for i, (h, t) in enumerate(((hq, tq), (hkv, tk), (hkv, tk))))
    else:
        Q, K, V = normal((tq, hq, d), dtype, seed, qstd), normal((tk, hkv, d), dtype, seed + 1), normal((tk, hkv, d), dtype, seed + 2)
    dO = normal((tq, hq, d), dtype, seed + 3)
    O, lse = torch.full((tq, hq, d), math.nan, dtype=dtype, device="cuda"), torch.full((hq, tq), math.nan, device="cuda")
    gq, gk = gpu_i32(cq), gpu_i32(ck)
    need = s24.attn_fwd_workspace(tq, tk, hq, hkv, d, len(lq))
    s24.attn_fwd(Q, K, V, O, lse, torch.empty(need, dtype=torch.uint8, device="cuda"), gq, gk, causal, scale)
    ref, bound = packed(Q, K, V, cq, ck, d ** -0.5 if scale is None else scale, causal, dO if backward else None)
    what = f"lq {lq} lk {lk} heads {hq}/{hkv} d {d} {dtype} causal {causal}"
    assert_within(O, ref["O"], bound["O"], f"O, {what}")
    assert_within(lse, ref["lse"], bound["lse"], f"lse, {what}")
    if not backward:
        return
    work = torch.empty(s24.attn_bwd_workspace(tq, tk, hq, hkv, d, len(lq)), dtype=torch.uint8, device="cuda")
    grads = [torch.full(x.shape, math.nan, dtype=dtype, device="cuda") for x in (Q, K, V)]
    s24.attn_bwd(Q, K, V, O, dO, lse, *grads, work, gq, gk, causal, scale)
    for n, x in zip(("dQ", "dK", "dV"), grads):
        assert_within(x, ref[n], bound[n], f"{n}, {what}")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 191, 300])
def test_one_sequence_of_every_length_around_the_tiles(s24, n, d, dtype):
    run(s24, [n], [n], 2, 1, d, dtype, seed=n)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (4, 2), (8, 8), (12, 4), (16, 2), (5, 5)])
def test_grouped_heads(s24, hq, hkv):
    run(s24, [70, 130], [70, 130], hq, hkv, 64, BF16, seed=hq)


@pytest.mark.parametrize("d", [16, 32, 48, 80, 96, 112])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_head_sizes_between(s24, d, dtype):
    run(s24, [90, 3], [90, 3], 4, 2, d, dtype, seed=d)


@pytest.mark.parametrize("views", ["projection", "heads", "dense"])
def test_strides(s24, views):
    run(s24, [100, 29], [100, 29], 4, 2, 128, BF16, views=views, seed=7)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([1], [200]), ([40], [300]), ([130], [131]), ([5, 70, 1], [64, 500, 1]), ([200], [40]), ([130, 10], [1, 9]), ([3, 50], [0, 60]),
                                   ([0, 33], [12, 33]), ([7], [0])])
def test_queries_and_keys_of_different_lengths(s24, lq, lk, causal):
    """Chunks of a prompt; more queries than keys, whose first rows see nothing when causal; sequences without queries or keys."""
    run(s24, lq, lk, 4, 2, 64, BF16, causal=causal, seed=len(lq))
    run(s24, lq, lk, 2, 2, 128, F16, causal=causal, seed=len(lq), backward=True)


def test_many_short_sequences(s24):
    rng = random.Random(3)
    lens = [rng.choice([0, 1, 2, 3, 17, 64, 65, 130]) for _ in range(150)]
    run(s24, lens, lens, 2, 1, 64, BF16, seed=5)


@pytest.mark.parametrize("d", [64, 128])
def test_large_scores(s24, d):
    """Scores far apart: the running reference moves, and most weights vanish."""
    run(s24, [333], [333], 2, 2, d, BF16, scale=1.0, seed=11, qstd=4.0)
    run(s24, [333], [333], 2, 2, d, F16, scale=1e-3, seed=12)


def test_growing_scores(s24):
    """Each key scores higher than the last, by less and by more than what moves the reference."""
    n, d = 400, 64
    for step in (0.02, 0.5):
        Q, K, V = torch.zeros((n, 1, d), dtype=BF16), torch.zeros((n, 1, d), dtype=BF16), normal((n, 1, d), BF16, 1)
        Q[:, 0, 0], K[:, 0, 0], K[:, 0, 1], Q[:, 0, 1] = 1.0, (torch.arange(n) * step).to(BF16), (torch.arange(n) * step - (torch.arange(n) * step).to(BF16)).to(BF16), 1.0
        Q, K = Q.cuda(), K.cuda()
        O, lse = torch.empty_like(Q), torch.empty((1, n), device="cuda")
        s24.attn_fwd(Q, K, V, O, lse, torch.empty(s24.attn_fwd_workspace(n, n, 1, 1, d, 1), dtype=torch.uint8, device="cuda"), gpu_i32([0, n]), None, True, 1.0)
        ref, bound = packed(Q, K, V, [0, n], [0, n], 1.0, True)
        assert_within(O, ref["O"], bound["O"], "O")
        assert_within(lse, ref["lse"], bound["lse"], "lse")


def test_other_sequences_do_not_reach_a_result(s24):
    """NaN and infinities in the sequences before and after, in rows of no sequence and in the gaps between heads."""
    lens = [50, 77, 40]
    cu = offsets(lens)
    n, hq, hkv, d = cu[-1] + 30, 4, 2, 64
    wide = normal((n, hq + 2 * hkv + 1, d), BF16, 4)
    clean = wide.clone()
    for bad in (math.nan, math.inf):
        wide[:cu[1]], wide[cu[2]:], wide[:, -1] = bad, bad, bad
        outs = []
        for x in (clean, wide):
            Q, K, V = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:-1]
            O, lse = torch.zeros((n, hq, d), dtype=BF16, device="cuda"), torch.zeros((hq, n), device="cuda")
            s24.attn_fwd(Q, K, V, O, lse, torch.empty(s24.attn_fwd_workspace(n, n, hq, hkv, d, 3), dtype=torch.uint8, device="cuda"), gpu_i32(cu))
            dO = normal((n, hq, d), BF16, 9)
            if x is wide:
                dO[:cu[1]], dO[cu[2]:] = bad, bad
            grads = [torch.zeros(t.shape, dtype=BF16, device="cuda") for t in (Q, K, V)]
            work = torch.empty(s24.attn_bwd_workspace(n, n, hq, hkv, d, 3), dtype=torch.uint8, device="cuda")
            s24.attn_bwd(Q, K, V, O, dO, lse, *grads, work, gpu_i32(cu))
            outs.append([t[cu[1]:cu[2]] for t in (O, *grads)] + [lse[:, cu[1]:cu[2]]] + [t[cu[-1]:] for t in (O, *grads)])
        for a, b in zip(*outs):
            assert torch.equal(a, b)


def test_gradients_against_differences(s24):
    """The gradient of sum(O * W) along random directions, against central differences of the 64-bit forward pass at the same point."""
    lens, hq, hkv, d = [37, 12], 4, 2, 64
    cu = offsets(lens)
    x = {n: normal((cu[-1], h, d), F16, i) for i, (n, h) in enumerate((("Q", hq), ("K", hkv), ("V", hkv), ("W", hq)))}
    O, lse = torch.empty_like(x["Q"]), torch.empty((hq, cu[-1]), device="cuda")
    s24.attn_fwd(x["Q"], x["K"], x["V"], O, lse, None, gpu_i32(cu))
    grads = {n: torch.empty_like(x[n]) for n in "QKV"}
    work = torch.empty(s24.attn_bwd_workspace(cu[-1], cu[-1], hq, hkv, d, 2), dtype=torch.uint8, device="cuda")
    s24.attn_bwd(x["Q"], x["K"], x["V"], O, x["W"], lse, grads["Q"], grads["K"], grads["V"], work, gpu_i32(cu))
    _, bound = packed(x["Q"], x["K"], x["V"], cu, cu, d ** -0.5, True, x["W"])
    y = {n: t.cpu().double() for n, t in x.items()}

    def loss(moved):
        total = 0.0
        for i in range(len(lens)):
            s = slice(cu[i], cu[i + 1])
            for h in range(hq):
                q, k, v = moved["Q"][s, h], moved["K"][s, h // 2], moved["V"][s, h // 2]
                t = (q @ k.T * d ** -0.5).masked_fill(torch.triu(torch.ones(len(q), len(q), dtype=torch.bool), 1), -math.inf)
                total += (torch.softmax(t, 1) @ v * moved["W"][s, h]).sum().item()
        return total

    for n in "QKV":
        way = torch.randn(y[n].shape, generator=torch.Generator().manual_seed(ord(n)), dtype=torch.float64)
        step = 1e-4
        slope = (loss(y | {n: y[n] + step * way}) - loss(y | {n: y[n] - step * way})) / (2 * step)
        got = (grads[n].cpu().double() * way).sum().item()
        assert abs(got - slope) <= (bound["d" + n] * way.abs()).sum().item() + 1e-5 * abs(slope)


def test_same_bits_every_time(s24):
    from paper_2404_01847_amd.attention import Attention
    lens = [700, 33, 513]
    cu = gpu_i32(offsets(lens))
    n = sum(lens)
    layer = Attention(16, 2, 128, n, dtype=BF16)
    x = normal((n, 20, 128), BF16, 3)
    Q, K, V, dO = x[:, :16], x[:, 16:18], x[:, 18:], normal((n, 16, 128), BF16, 4)
    first = None
    for _ in range(4):
        out = [t.clone() for t in (layer.forward(Q, K, V, cu), *layer.backward(Q, K, V, dO, cu))]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))


# ---------------------------------------------------------------------------------------------------- cache
def filled(s24, lens, page, hkv, d, dtype, bits, seed=0, vstd=1.0, spare=3):
    """A cache whose unused places hold NaN (8 bits: NaN steps), its table, and what was written."""
    from paper_2404_01847_amd.attention import PagedKV
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), max(max(counts), 1)), 0x7FFFFFFF, dtype=torch.int32)   # entries past a sequence's pages hold anything
    places, at = [], 0
    for i, (n, k) in enumerate(zip(lens, counts)):
        table[i, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        places += [order[at + j // page] * page + j % page for j in range(n)]
        at += k
    cache = PagedKV(pages, page, hkv, d, dtype, bits=bits)
    for t in (cache.K, cache.V):
        t.fill_(255 if bits == 8 else math.nan)
    for t in (cache.k_step, cache.v_step) if bits == 8 else ():
        t.fill_(math.nan)
    n = sum(lens)
    K, V = normal((n, hkv, d), dtype, seed + 1), normal((n, hkv, d), dtype, seed + 2, vstd)
    cache.write(K, V, torch.tensor(places, dtype=torch.int64, device="cuda"))
    return cache, table.cuda(), K, V


def held(x, bits):
    if bits == 16:
        return x.cpu().double()
    n, s = quantise(x)
    return n * s


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,hkv,page", [(64, 3, 16), (128, 2, 64), (80, 1, 32), (16, 2, 128), (112, 2, 256)])
def test_cache_reads_back_what_was_written(s24, d, hkv, page, dtype, bits):
    lens = [1, 17, 0, 64, 200, 33]
    cache, table, K, V = filled(s24, lens, page, hkv, d, dtype, bits, seed=d)
    cu = gpu_i32(offsets(lens))
    Ko, Vo = torch.full_like(K, math.nan), torch.full_like(V, math.nan)
    cache.read(table, cu, Ko, Vo)
    for got, x in ((Ko, K), (Vo, V)):
        want = x.cpu().double() if bits == 16 else held(x, 8).float().to(dtype).double()    # s*n in fp32, then rounded
        assert torch.equal(got.cpu().double(), want)


def test_quantised_exactly_where_the_quotient_is_close_to_a_tie(s24):
    """Every bf16 value of some binades against steps of many kinds: the numbers are those of 64 bits, ties to even."""
    from paper_2404_01847_amd.attention import PagedKV
    for dtype in (BF16, F16):
        every = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(dtype)
        every = every[every.float().isfinite()]
        most = (every.float().abs() + 0).sort().values
        rows = []
        for i in range(4000):      # a row's largest value, and 15 that lie near odd multiples of half its step
            top = most[(i * 7919) % len(most)].float().item()
            half = max(top / 127, 2.0 ** -126) / 2
            rows.append([top] + [half * (2 * ((i + 9 * j) % 127) + 1) * (-1) ** j for j in range(15)])
        x = torch.tensor(rows).to(dtype).view(-1, 1, 16).cuda()
        x = torch.where(x.isfinite(), x, torch.zeros_like(x))
        n = x.shape[0]
        cache = PagedKV(n // 16, 16, 1, 16, dtype, bits=8)
        cache.write(x, x, torch.arange(n, device="cuda"))
        want, step = quantise(x)
        assert torch.equal(cache.k_step.flatten().cpu().double(), step.flatten()) and torch.equal(cache.v_step.flatten().cpu().double(), step.flatten())
        assert torch.equal(cache.K.flatten(0, 2).cpu().double() - 128, want[:, 0])
        assert torch.equal(cache.V.reshape(n // 16, 16, 16).transpose(1, 2).reshape(n, 16).cpu().double() - 128, want[:, 0])


def test_zero_rows_and_skipped_places(s24):
    from paper_2404_01847_amd.attention import PagedKV
    cache = PagedKV(2, 16, 2, 64, BF16, bits=8)
    for t in (cache.K, cache.V, cache.k_step, cache.v_step):
        t.zero_()
    K = normal((4, 2, 64), BF16, 1)
    K[1] = 0
    cache.write(K, K, torch.tensor([3, 4, -1, 32], device="cuda"))     # the last two: padding, and past the cache
    torch.cuda.synchronize()
    assert int((cache.k_step != 0).sum()) == 4 and int((cache.K[0, :, 4] == 128).all())
    assert int(cache.K[1].sum()) == 0 and int(cache.K[0, :, :3].sum()) == 0 and int(cache.K[0, :, 5:].sum()) == 0


def decode(s24, lens, hq, hkv, d, dtype, bits, page, scale=None, seed=0, vstd=1.0, qstd=1.0):
    cache, table, K, V = filled(s24, lens, page, hkv, d, dtype, bits, seed, vstd)
    Q = normal((len(lens), hq, d), dtype, seed + 5, qstd)
    O = torch.full_like(Q, math.nan)
    cache.attend(Q, table, gpu_i32(lens), O, scale)
    scale = d ** -0.5 if scale is None else scale
    Kh, Vh, q, cu, u = held(K, bits), held(V, bits), Q.cpu().double(), offsets(lens), U[dtype]
    ref, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for i, n in enumerate(lens):
        if n == 0:
            continue
        for h in range(hq):
            k, v = Kh[cu[i]:cu[i + 1], h // (hq // hkv)], Vh[cu[i]:cu[i + 1], h // (hq // hkv)]
            P = torch.softmax(k @ q[i, h] * scale, 0)
            e = d * 2.0 ** -24 * (k.abs() @ q[i, h].abs() * scale).max() + 2.0 ** -20
            weights = 2.0 ** -11 if bits == 8 else u       # rounding of the weights, and what is lost of the smallest:
            lost = 2.0 ** -25 * n * (4 * 127 * quantise(V[cu[i]:cu[i + 1], h // (hq // hkv)])[1].max() if bits == 8 else 0.0) + \
                OPERAND_TINY[dtype] * n * v.abs().max()
            ref[i, h] = P @ v
            bound[i, h] = u * ref[i, h].abs() + (weights + 2 * e) * (P @ v.abs()) + lost + TINY[dtype]
    assert_within(O, ref, bound, f"lens {lens} heads {hq}/{hkv} d {d} {dtype} bits {bits} page {page}")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1], [0], [15, 16, 17], [63, 64, 65], [0, 255, 256, 257, 0], [1000, 3, 511]])
def test_decode_lengths(s24, lens, d, dtype, bits):
    decode(s24, lens, 4, 2, d, dtype, bits, 16, seed=sum(lens))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (15, 1), (17, 1), (40, 2), (5, 5), (64, 8)])
def test_decode_grouped_heads(s24, hq, hkv, bits):
    decode(s24, [300, 40], hq, hkv, 64, BF16, bits, 32, seed=hq)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [16, 32, 48, 80, 96, 112])
def test_decode_head_sizes_between(s24, d, bits):
    decode(s24, [70, 300], 4, 2, d, F16, bits, 64, seed=d)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 512])
@pytest.mark.parametrize("bits", [16, 8])
def test_decode_pages(s24, page, bits):
    decode(s24, [20, 700, 129], 2, 2, 128, BF16, bits, page, seed=page)


@pytest.mark.parametrize("bits", [16, 8])
def test_decode_many_tiles(s24, bits):
    """Long enough to be split, among short ones."""
    decode(s24, [30000, 5, 2000, 0, 70], 2, 1, 64, BF16, bits, 64, seed=2)


@pytest.mark.parametrize("bits", [16, 8])
def test_decode_many_sequences(s24, bits):
    rng = random.Random(1)
    decode(s24, [rng.choice([0, 1, 5, 70, 300]) for _ in range(200)], 2, 2, 64, BF16, bits, 16, seed=2)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("vstd,qstd", [(1e-5, 1.0), (1e4, 1.0), (1.0, 30.0), (1.0, 1e-6)])
def test_decode_scales_of_the_data(s24, vstd, qstd, bits):
    decode(s24, [600], 4, 2, 64, BF16, bits, 16, seed=3, vstd=vstd, qstd=qstd)


def test_decode_length_beyond_the_table_is_cut(s24):
    cache, table, K, V = filled(s24, [32], 16, 1, 64, BF16, 16)
    Q = normal((1, 1, 64), BF16, 1)
    a, b = torch.empty_like(Q), torch.empty_like(Q)
    cache.attend(Q, table, gpu_i32([32]), a)
    cache.attend(Q, table, gpu_i32([5000]), b)
    cache.attend(Q, table, gpu_i32([-3]), Q)
    assert torch.equal(a, b) and int((Q != 0).sum()) == 0


def test_decode_in_a_graph_on_another_stream(s24):
    """The write of a token and its attention, captured and replayed with new lengths in the same buffers."""
    lens = [300, 20, 700]
    cache, table, K, V = filled(s24, lens, 16, 2, 64, BF16, 8)
    Q, n = normal((3, 4, 64), BF16, 1), gpu_i32(lens)
    O, want = torch.empty_like(Q), torch.empty_like(Q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.attend(Q, table, n, O)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.attend(Q, table, n, O)
    for cut in (0, 1, 100, 19):
        n.copy_(gpu_i32([max(0, x - cut) for x in lens]))
        Q.copy_(normal((3, 4, 64), BF16, cut))
        O.fill_(math.nan)
        graph.replay()
        cache.attend(Q, table, n, want)
        torch.cuda.synchronize()
        assert torch.equal(O, want)


def test_a_prompt_in_chunks_gives_what_the_whole_gives(s24):
    """Prompt, cache and sampling together: the chunks of a prompt attend to what is read back, the last token through the pages."""
    from paper_2404_01847_amd.attention import Attention, PagedKV
    n, hq, hkv, d, page = 333, 4, 2, 64, 32
    x = normal((n, hq + 2 * hkv, d), BF16, 1)
    Q, K, V = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    whole = Attention(hq, hkv, d, n).forward(Q, K, V, gpu_i32([0, n]))
    cache = PagedKV(11, page, hkv, d)
    table = torch.randperm(11, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None]
    at = torch.arange(n, device="cuda")
    places = table[0].long()[at // page] * page + at % page
    ref, bound = packed(Q, K, V, [0, n], [0, n], d ** -0.5, True)
    for a, b in ((0, 100), (100, 101), (101, 333)):
        cache.write(K[a:b], V[a:b], places[a:b])
        Kb, Vb = (torch.empty((b, hkv, d), dtype=BF16, device="cuda") for _ in range(2))
        cache.read(table, gpu_i32([0, b]), Kb, Vb)
        assert torch.equal(Kb, K[:b]) and torch.equal(Vb, V[:b])
        out = Attention(hq, hkv, d, b - a, b).forward(Q[a:b], Kb, Vb, gpu_i32([0, b - a]), gpu_i32([0, b]))
        assert_within(out, ref["O"][a:b], bound["O"][a:b], f"chunk {a}:{b}")
    O = torch.empty((1, hq, d), dtype=BF16, device="cuda")
    cache.attend(Q[-1:].contiguous(), table, gpu_i32([n]), O)
    assert_within(O, ref["O"][-1:], bound["O"][-1:], "last token")
    assert_within(whole, ref["O"], bound["O"], "whole")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d,hkv", [(64, 5), (64, 12), (128, 8), (80, 3), (16, 4)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_many_tokens_of_sequences_that_start_anywhere(s24, d, hkv, dtype, bits):
    """Enough tokens for the kernel that takes runs: continued sequences of odd lengths, single tokens, padding between them, tokens out of order; what was
    in the pages stays."""
    from paper_2404_01847_amd.attention import PagedKV
    rng, page = random.Random(d + bits), 32
    past = [rng.choice([0, 1, 15, 16, 17, 40]) for _ in range(400)]
    new = [rng.choice([1, 2, 15, 16, 17, 31, 100, 130]) for _ in past]
    lens = [a + b for a, b in zip(past, new)]
    counts = [-(-n // page) for n in lens]
    order = list(range(sum(counts)))
    rng.shuffle(order)
    table, places, at = torch.zeros((len(lens), max(counts)), dtype=torch.int32), [], 0
    for i, k in enumerate(counts):
        table[i, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        places.append([order[at + j // page] * page + j % page for j in range(lens[i])])
        at += k
    cu, n = offsets(lens), sum(lens)
    K, V = normal((n, hkv, d), dtype, 1), normal((n, hkv, d), dtype, 2)
    cache = PagedKV(len(order), page, hkv, d, dtype, bits=bits)
    flat = torch.tensor([p for x in places for p in x], dtype=torch.int64, device="cuda")
    old = torch.tensor([j < past[i] for i in range(len(lens)) for j in range(lens[i])], device="cuda")
    cache.write(K[old].contiguous(), V[old].contiguous(), flat[old].contiguous())
    rows = torch.nonzero(~old)[:, 0]
    half = len(rows) // 2
    back = rows[half:half + 1000].flip(0)                       # some of the tokens come in descending order
    rows = torch.cat([rows[:half], back, rows[half + 1000:]])
    gaps = torch.full((len(rows) * 2,), -1, dtype=torch.int64, device="cuda")
    keep = torch.ones(len(gaps), dtype=torch.bool, device="cuda")
    keep[2 * half - 3000:2 * half] = False                      # padding among them: every second row there
    index = torch.arange(len(rows), device="cuda")
    index = index + torch.clamp(index - (half - 500), 0, 1000)
    K2, V2 = (torch.full((int(index.max()) + 8, hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    to = gaps[:K2.shape[0]].clone()
    K2[index], V2[index], to[index] = K[rows], V[rows], flat[rows]
    to[-1] = len(order) * page + 5
    cache.write(K2, V2, to)
    Ko, Vo = torch.full_like(K, math.nan), torch.full_like(V, math.nan)
    cache.read(table.cuda(), gpu_i32(cu), Ko, Vo)
    for got, x in ((Ko, K), (Vo, V)):
        assert torch.equal(got.cpu().double(), x.cpu().double() if bits == 16 else held(x, 8).float().to(dtype).double())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_runs_are_quantised_as_single_tokens_are(s24, dtype):
    """The same values through both kernels of the cache: the same bytes and steps, also for values on and beside ties."""
    from paper_2404_01847_amd.attention import PagedKV
    n, hkv, d = 20000, 4, 128
    x = normal((n, hkv, d), dtype, 1)
    top = x.abs().amax(2, keepdim=True).float()
    ties = ((torch.arange(n * hkv * d, device="cuda").view(n, hkv, d) % 127 + 0.5) * top / 127).to(dtype)
    x[::2, :, 1:] = torch.where(ties[::2, :, 1:].abs() <= top[::2], ties[::2, :, 1:], x[::2, :, 1:])
    one, two = (PagedKV(n // 16, 16, hkv, d, dtype, bits=8) for _ in range(2))
    at = torch.arange(n, device="cuda")
    one.write(x, x, at)
    for i in range(0, n, 50):
        two.write(x[i:i + 50], x[i:i + 50], at[i:i + 50])
    for a, b in zip((one.K, one.V, one.k_step, one.v_step), (two.K, two.V, two.k_step, two.v_step)):
        assert torch.equal(a, b)
    want, _ = quantise(x)
    assert torch.equal(one.K.transpose(1, 2).reshape(n, hkv, d).cpu().double() - 128, want)


def test_offsets_past_32_bits(s24):
    """Heads that lie 2^31 values apart, and pages beyond 2^32 bytes."""
    n, d, gap = 70, 64, 1 << 31
    flat = torch.empty(gap + n * d, dtype=BF16, device="cuda")
    apart = lambda: flat.as_strided((n, 2, d), (d, gap, 1))
    values = [normal((n, 2, d), BF16, i) for i in range(4)]
    cu, grads = gpu_i32([0, n]), {}
    for far in (None, 0, 1, 2, 3):
        x = list(values)
        if far is not None:
            apart().copy_(x[far])
            x[far] = apart()
        Q, K, V, dO = x
        O, lse = torch.empty_like(values[0]), torch.empty((2, n), device="cuda")
        s24.attn_fwd(Q, K, V, O, lse, None, cu)
        out = [torch.empty_like(values[0]) for _ in range(3)]
        work = torch.empty(s24.attn_bwd_workspace(n, n, 2, 2, d, 1), dtype=torch.uint8, device="cuda")
        s24.attn_bwd(Q, K, V, O, dO, lse, *out, work, cu)
        grads[far] = [O, *out]
    for far in (0, 1, 2, 3):
        assert all(torch.equal(a, b) for a, b in zip(grads[None], grads[far]))
    s24.attn_fwd(*values[:3], apart(), None, None, cu)
    assert torch.equal(apart(), grads[None][0])
    del flat
    from paper_2404_01847_amd.attention import PagedKV
    for bits, pages in ((16, 70000), (8, 140000)):
        cache = PagedKV(pages, 64, 8, 64, bits=bits)
        assert cache.K.numel() * cache.K.element_size() > 1 << 32
        K, V, Q = (normal((300, 8, 64), BF16, i) for i in range(3))
        table = (pages - 1 - torch.arange(5, dtype=torch.int32, device="cuda"))[None]
        at = torch.arange(300, device="cuda")
        cache.write(K, V, table[0].long()[at // 64] * 64 + at % 64)
        small, low = PagedKV(5, 64, 8, 64, bits=bits), torch.arange(5, dtype=torch.int32, device="cuda")[None]
        small.write(K, V, at)
        outs = []
        for c, t in ((cache, table), (small, low)):
            Ko, Vo, O = torch.empty_like(K), torch.empty_like(V), torch.empty_like(Q[:1])
            c.read(t, gpu_i32([0, 300]), Ko, Vo)
            c.attend(Q[:1], t, gpu_i32([300]), O)
            outs.append((Ko, Vo, O))
        assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_offsets_and_tables_that_hold_anything_stay_in_the_operands(s24):
    """Offsets that do not ascend and page numbers that do not exist are cut to what there is: no result is promised, none is touched that is not theirs."""
    n, hq, hkv, d = 100, 2, 1, 64
    Q, K, V = normal((n, hq, d), BF16, 1), normal((n, hkv, d), BF16, 2), normal((n, hkv, d), BF16, 3)
    O, lse = torch.zeros_like(Q), torch.zeros((hq, n), device="cuda")
    work = torch.empty(max(s24.attn_bwd_workspace(n, n, hq, hkv, d, 3), s24.attn_fwd_workspace(n, n, hq, hkv, d, 3)), dtype=torch.uint8, device="cuda")
    grads = [torch.zeros_like(x) for x in (Q, K, V)]
    for bad in ([0, 1 << 30, 50, 100], [-5, 20, -7, 300], [90, 80, 70, 60], [0, 100, 100, 2 ** 31 - 1]):
        for cq, ck in ((bad, bad), (bad, [0, 30, 60, 100]), ([0, 30, 60, 100], bad)):
            s24.attn_fwd(Q, K, V, O, lse, work, gpu_i32(cq), gpu_i32(ck))
            s24.attn_bwd(Q, K, V, O, Q, lse, *grads, work, gpu_i32(cq), gpu_i32(ck))
    cache, table, K, V = filled(s24, [40, 40], 16, 1, 64, BF16, 16)
    O = torch.empty_like(Q[:2])
    table.fill_(-1)
    cache.attend(Q[:2], table, gpu_i32([40, 1000000]), O)
    cache.read(table, gpu_i32([30, -4, 200]), K, V)
    cache.write(K, V, torch.randint(-(1 << 40), 1 << 40, (80,), device="cuda"))
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------------------------------- values that are no numbers, and extreme scores
@pytest.mark.parametrize("n", [33, 2000])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_the_8_bit_cache_does_not_lose_what_is_no_number(s24, bad, n):
    """Such a token's head has the step NaN: it reads back as NaN, and its sequence's attention is NaN; others stay."""
    from paper_2404_01847_amd.attention import PagedKV
    pages = -(-n // 16)
    cache = PagedKV(2 * pages, 16, 8, 128, BF16, bits=8)
    K, V = normal((2 * 16 * pages, 8, 128), BF16, 1), normal((2 * 16 * pages, 8, 128), BF16, 2)
    K[5, 3, 17] = bad
    V[9, 6, 100] = bad
    cache.write(K, V, torch.arange(2 * 16 * pages, device="cuda"))
    steps_k, steps_v = (t.transpose(1, 2).reshape(-1, 8) for t in (cache.k_step, cache.v_step))
    assert steps_k.isnan().nonzero().tolist() == [[5, 3]] and steps_v.isnan().nonzero().tolist() == [[9, 6]]
    table = torch.arange(2 * pages, dtype=torch.int32, device="cuda").view(2, pages)
    Ko, Vo = torch.empty((2 * n, 8, 128), dtype=BF16, device="cuda"), torch.empty((2 * n, 8, 128), dtype=BF16, device="cuda")
    cache.read(table, gpu_i32([0, n, 2 * n]), Ko, Vo)
    assert Ko.isnan().all(2).nonzero().tolist() == [[5, 3]] and int(Ko.isnan().sum()) == 128
    assert Vo.isnan().all(2).nonzero().tolist() == [[9, 6]] and int(Vo.isnan().sum()) == 128
    Q = normal((2, 16, 128), BF16, 3)
    O = torch.zeros_like(Q)
    cache.attend(Q, table, gpu_i32([n, n]), O)
    assert O[0, 6:8].isnan().all() and O[0, 12:14].isnan().all() and int(O.isnan().sum()) == 4 * 128


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,heads", [(70, 2), (3000, 1)])     # in one part, and in several
def test_what_is_no_number_shows_in_the_statistics_and_gradients(s24, n, heads, d):
    from paper_2404_01847_amd.attention import Attention
    cu = gpu_i32([0, n])
    layer = Attention(heads, heads, d, n, n, BF16)
    Q, K, V, dO = (normal((n, heads, d), BF16, i) for i in range(4))
    K[40, 0, 3] = math.nan                                      # queries from 40 on see it
    layer.forward(Q, K, V, cu)
    dQ = layer.backward(Q, K, V, dO, cu)[0]
    assert layer.lse[0, 40:].isnan().all() and layer.lse[0, :32].isfinite().all() and layer.lse[1:].isfinite().all()
    assert layer.O[40:, 0].isnan().all() and dQ[40:, 0].isnan().all() and layer.O[:, 1:].isfinite().all() and dQ[:, 1:].isfinite().all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("sign", [-1, 1])
def test_equal_scores_of_any_size_weigh_the_same(s24, bits, sign):
    """All of a row's scores are 2^23 or its negative.  The weights are then one number, which the second product has rounded to its type: 2^-8, or 2^-11 with a
    token's step, of the weighted sizes; the result's rounding is another 2^-8 of it."""
    from paper_2404_01847_amd.attention import Attention
    n, d = 300, 64
    K, Q = torch.full((n, 1, d), sign * 2.0 ** 9, dtype=BF16, device="cuda"), torch.full((n, 1, d), 2.0 ** 11, dtype=BF16, device="cuda")
    V = normal((n, 1, d), BF16, 1)

    def bound(mean, size, weights):
        return 2.0 ** -8 * mean.abs() + (1 + 2.0 ** -8) * (weights + 2.0 ** -13) * size
    if bits == 16:
        layer, count = Attention(1, 1, d, n, n, BF16), torch.arange(1, n + 1, device="cuda").view(-1, 1, 1)
        O = layer.forward(Q, K, V, gpu_i32([0, n]))
        mean, size = V.double().cumsum(0) / count, V.double().abs().cumsum(0) / count
        assert ((O.double() - mean).abs() <= bound(mean, size, 2.0 ** -8)).all()
    cache, table, _, _ = filled(s24, [n], 32, 1, d, BF16, bits)
    cache.write(K, V, table[0].long().repeat_interleave(32)[:n] * 32 + torch.arange(n, device="cuda") % 32)
    O = torch.full((1, 1, d), math.nan, dtype=BF16, device="cuda")
    cache.attend(Q[:1], table, gpu_i32([n]), O)
    x = held(V, bits).cuda()
    assert ((O[0].double() - x.mean(0)).abs() <= bound(x.mean(0), x.abs().mean(0), 2.0 ** -11 if bits == 8 else 2.0 ** -8)).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("count", [2, 31, 64, 65])     # a wave holds the lengths of 64
def test_tiles_of_many_sequences_are_all_taken(s24, count, causal):
    """Tiles go by their length, whatever sequence they are of; empty sequences, and some with more keys or more queries, among them."""
    rng = random.Random(count)
    lk = [rng.choice([0, 1, 20, 129, 400, rng.randrange(1, 700)]) for _ in range(count - 1)] + [650]
    lq = [rng.choice([n, n, n, n // 2, n + rng.choice([0, 140])]) for n in lk]
    run(s24, lq, lk, 2, 1, 64, BF16, causal=causal, seed=count)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("count", [64, 65, 256, 257, 600])
def test_decode_shares_of_many_sequences(s24, count, bits):
    """One long sequence, so that the shares do not go by sequences, among short and empty ones, also at either end."""
    rng = random.Random(count)
    lens = [rng.choice([0, 0, 1, 5, 64, 65, 130]) for _ in range(count)]
    for at in (0, count // 2, count - 1):
        run = list(lens)
        run[at] = 700
        decode(s24, run, 2, 1, 64, BF16, bits, 32, seed=at)
    decode(s24, [0] * (count - 1) + [600], 2, 1, 64, BF16, bits, 32, seed=1)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("longest", [16, 128, 129, 512, 513])
def test_decode_sequences_short_enough_for_one_wave(s24, longest, bits):
    """With few sequences up to 128 positions, with many up to 512; some are empty."""
    rng = random.Random(longest)
    for count, hq, hkv in ((5, 20, 1), (90, 34, 34)):
        lens = [rng.choice([0, 1, longest // 2, longest]) for _ in range(count - 1)] + [longest]
        decode(s24, lens, hq, hkv, 64, BF16, bits, 16, seed=longest)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("lens,heads", [([2, 3, 5, 8, 13, 21, 34, 1], (6, 3)), ([700], (1, 1)), ([9000], (4, 1))])     # few tiles; several parts; a launch for each gradient
def test_gradients_are_about_as_exact_as_their_own_rounding(s24, lens, heads, d, dtype):
    """In the 2-norm, against results of 64 bits that are rounded once.  dS is in 16 bits or more, delta in 15, P (of dV) in the type's: its rounding, which no sum
    makes larger than the result's own, allows dV the square root of two; a fifth more for what is left of the others."""
    from paper_2404_01847_amd.attention import Attention
    (hq, hkv), n = heads, sum(lens)
    if n == 9000:
        lens, hq, hkv, n = [300] * 30, 16, 16, 9000
    cu = offsets(lens)
    layer = Attention(hq, hkv, d, n, n, dtype)
    Q, K, V, dO = normal((n, hq, d), dtype, 1), normal((n, hkv, d), dtype, 2), normal((n, hkv, d), dtype, 3), normal((n, hq, d), dtype, 4)
    K = (K.float() * torch.exp(0.5 * torch.randn((1, hkv, d), generator=torch.Generator().manual_seed(5))).cuda()).to(dtype)
    layer.forward(Q, K, V, gpu_i32(cu))
    grads = layer.backward(Q, K, V, dO, gpu_i32(cu))
    ref, _ = packed(Q, K, V, cu, cu, d ** -0.5, True, dO)
    for name, got in zip(("dQ", "dK", "dV"), grads):
        want = ref[name].reshape(got.shape)
        off, own = (got.cpu().double() - want).norm(), (want.to(dtype).double() - want).norm()
        assert off <= (1.7 if name == "dV" else 1.2) * own, (name, (off / own).item())


def test_a_rest_of_the_wrong_kind_is_refused(s24):
    x, cu = normal((8, 2, 64), BF16, 1), gpu_i32([0, 8])
    for rest in (torch.empty((8, 2, 64), dtype=torch.uint8, device="cuda"), torch.empty((8, 2, 32), dtype=torch.int8, device="cuda"), torch.empty((8, 2, 64), dtype=torch.int8)):
        with pytest.raises(ValueError, match="rest"):
            s24.attn_fwd(x, x, x, torch.empty_like(x), None, None, cu, rest=rest)
