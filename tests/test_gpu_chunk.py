"""Attention of new tokens over the paged cache, on the GPU against 64 bits on the CPU with the bounds of attention_reference.py."""
import math

import pytest
import torch

from attention_reference import OPERAND_TINY, TINY, U, assert_within, quantise, visible
from test_gpu_attention import filled, gpu_i32, held, normal, offsets

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def reference(Q, K, V, new, lens, bits, scale, causal):
    """Results and bounds: roundings of the weights as operands (binary16 in an 8-bit cache) and of the result, the scores' error, and the smallest weights that are lost."""
    dtype, (_, hq, d), hkv = Q.dtype, Q.shape, K.shape[1]
    Kh, Vh, q, u = held(K, bits), held(V, bits), Q.cpu().double(), U[Q.dtype]
    a, b = offsets(new), offsets(lens)
    ref, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for i, (n, m) in enumerate(zip(new, lens)):
        if n == 0 or m == 0:
            continue
        seen, rows = visible(n, m, causal), slice(a[i], a[i + 1])
        steps = quantise(V[b[i]:b[i + 1]])[1][..., 0] if bits == 8 else None
        for h in range(hq):
            g = h // (hq // hkv)
            k, v = Kh[b[i]:b[i + 1], g], Vh[b[i]:b[i + 1], g]
            s = (q[rows, h] @ k.T * scale).masked_fill(~seen, -math.inf)
            P = torch.exp(s - torch.logsumexp(s, 1, keepdim=True)).masked_fill(~seen, 0.0)
            e = d * 2.0 ** -24 * (q[rows, h].abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True) + 2.0 ** -20
            weights = 2.0 ** -11 if bits == 8 else u
            lost = 2.0 ** -25 * m * 4 * 127 * steps[:, g].max() if bits == 8 else OPERAND_TINY[dtype] * 256 * m * v.abs().max()
            ref[rows, h] = P @ v
            bound[rows, h] = u * ref[rows, h].abs() + (weights + 2 * e) * (P @ v.abs()) + lost + TINY[dtype]
    return ref, bound


def chunk(new, lens, hq, hkv, d, dtype, bits, page, causal=True, scale=None, seed=0, vstd=1.0, qstd=1.0, views="whole"):
    cache, table, K, V = filled(None, lens, page, hkv, d, dtype, bits, seed, vstd)
    n = sum(new)
    if views == "projection":
        Q = normal((n, hq + 2 * hkv, d), dtype, seed + 5, qstd)[:, :hq]
    elif views == "heads":
        Q = normal((hq, n, d), dtype, seed + 5, qstd).transpose(0, 1)
    else:
        Q = normal((n, hq, d), dtype, seed + 5, qstd)
    O = torch.full((n, hq, d), math.nan, dtype=dtype, device="cuda")
    cache.attend_chunk(Q, gpu_i32(offsets(new)), table, gpu_i32(lens), O, scale, causal)
    ref, bound = reference(Q, K, V, new, lens, bits, d ** -0.5 if scale is None else scale, causal)
    assert_within(O, ref, bound, f"new {new} of {lens} heads {hq}/{hkv} d {d} {dtype} bits {bits} page {page} causal {causal}")
    return O


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200])
def test_whole_prompts_of_every_length_around_the_tiles(n, d, dtype, bits):
    chunk([n], [n], 2, 1, d, dtype, bits, 16)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([1], [200]), ([40], [300]), ([130], [131]), ([5, 70, 1], [64, 500, 1]), ([3, 0, 9], [50, 20, 9]), ([200], [40]), ([130, 10], [1, 9]),
                                      ([3, 50], [0, 60]), ([1, 1, 1, 1], [15, 16, 17, 700]), ([6] * 24, list(range(100, 1300, 50)))])
def test_new_tokens_after_others(new, lens, causal, bits):
    chunk(new, lens, 4, 2, 64, BF16, bits, 32, causal)
    chunk(new, lens, 4, 1, 128, F16, bits, 64, causal)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (8, 1), (17, 1), (5, 5), (40, 8), (64, 8), (12, 4), (130, 1)])
def test_grouped_heads(hq, hkv, bits):
    chunk([7, 30], [90, 33], hq, hkv, 64, BF16, bits, 16)


@pytest.mark.parametrize("bits", [16, 8])
def test_more_heads_than_the_device_holds_workgroups(bits):
    chunk([3, 40], [130, 900], 600, 600, 16, BF16, bits, 16)
    chunk([3, 1], [300, 500], 600, 600, 16, BF16, bits, 16)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [16, 32, 48, 80, 96, 112])
def test_head_sizes_between(d, bits):
    for dtype in (BF16, F16):
        chunk([40, 3], [150, 77], 4, 2, d, dtype, bits, 16)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 512])
def test_pages(page, bits):
    chunk([50, 20], [300, 129], 4, 2, 128, BF16, bits, page, seed=page)


@pytest.mark.parametrize("views", ["projection", "heads"])
def test_strides(views):
    chunk([50, 20], [300, 129], 6, 2, 64, BF16, 8, 32, views=views)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new,lens,heads,d", [([1], [6000], (8, 1), 128), ([5], [5000], (4, 2), 64), ([100], [4000], (2, 2), 128), ([3, 200, 1], [3000, 500, 2500], (4, 1), 96)])
def test_few_rows_over_many_positions(new, lens, heads, d, bits):
    """What a tile goes over is cut into parts."""
    chunk(new, lens, *heads, d, BF16, bits, 64)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("count", [2, 63, 64, 65, 200])
def test_many_sequences(count, bits):
    gen = torch.Generator().manual_seed(count)
    lens = torch.randint(1, 90, (count,), generator=gen).tolist()
    new = [min(n, int(torch.randint(0, 40, (1,), generator=gen))) for n in lens]
    chunk(new, lens, 4, 2, 64, BF16, bits, 16, seed=count)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new,lens", [([5] * 16, list(range(300, 460, 10))), ([1, 2, 33, 1, 0, 4], [700, 64, 500, 129, 300, 192]), ([2] * 90, [140 + 3 * i for i in range(90)]), ([7, 1], [703, 704]), ([3], [130])])
def test_short_sequences_of_few_rows(new, lens, bits):
    """None is cut, and there is no workspace."""
    import paper_2404_01847_amd as s24
    for heads, d, page in (((4, 2), 64, 64), ((8, 4), 112, 16)):
        chunk(new, lens, *heads, d, BF16, bits, page, seed=len(new))
        cache = filled(None, [16], page, heads[1], d, BF16, bits)[0]
        assert s24.attn_chunk_workspace(cache.buffers, 704 // page, sum(new), len(new), heads[0]) == 0


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("short,long,positions,heads", [(90, 10, 20000, 4), (60, 6, 5000, 7), (200, 50, 1200, 2), (249, 1, 30000, 2), (100, 27, 3000, 4), (300, 2, 10000, 1)])
def test_many_short_sequences_beside_long_ones(short, long, positions, heads, bits):
    """More sequences than lanes, most of them of one step, a few cut into parts."""
    gen = torch.Generator().manual_seed(short)
    lens = torch.randint(1, 64, (short,), generator=gen).tolist()
    for i in range(long):
        lens.insert(i * (len(lens) // long), positions - 7 * i)
    chunk([1 + (i % 9 == 0 and n > 1) for i, n in enumerate(lens)], lens, heads, heads, 16, BF16, bits, 64, seed=short)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new,lens,heads", [([33, 40, 1], [5000, 4800, 300], 128), ([33] * 5 + [2], [3000, 2900, 2800, 900, 70, 2000], 128), ([20, 3, 33], [4000, 4000, 4100], 256),
                                            ([33, 1] * 40 + [7] * 10, [6400] * 80 + [60] * 10, 4), ([1] * 150, [1500] * 75 + [3000] * 75, 4)])
def test_tiles_that_do_not_go_evenly_into_the_workgroups(new, lens, heads, bits):
    """They are cut into twice as many parts as the device holds at once."""
    chunk(new, lens, heads, heads, 16, F16, bits, 64, seed=len(new))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("vstd,qstd", [(1e-5, 1.0), (1e4, 1.0), (1.0, 30.0), (1.0, 1e-6)])
def test_scales_of_the_data(vstd, qstd, bits):
    chunk([20, 100], [500, 100], 4, 2, 128, BF16, bits, 32, vstd=vstd, qstd=qstd)


def test_steps_that_grow_along_a_sequence():
    """Values whose steps are larger by 2^20 in later tiles, and keys whose scores grow: the reference follows both."""
    from paper_2404_01847_amd.attention import PagedKV
    n, d, hq, hkv = 640, 64, 4, 2
    cache = PagedKV(40, 16, hkv, d, BF16, bits=8)
    growth = torch.exp2(torch.arange(n, device="cuda") * (20.0 / n))[:, None, None]
    K, V = normal((n, hkv, d), BF16, 1), (normal((n, hkv, d), BF16, 2).float() * growth * 1e-3).to(BF16)
    K = (K.float() * growth.sqrt().clamp(max=30)).to(BF16)
    cache.write(K, V, torch.arange(n, device="cuda"))
    Q, O = normal((100, hq, d), BF16, 3), torch.empty((100, hq, d), dtype=BF16, device="cuda")
    cache.attend_chunk(Q, gpu_i32([0, 100]), torch.arange(40, dtype=torch.int32, device="cuda")[None], gpu_i32([n]), O)
    ref, bound = reference(Q, K, V, [100], [n], 8, d ** -0.5, True)
    assert_within(O, ref, bound, "growing steps")


def test_single_tokens_agree_with_the_call_for_them():
    """One new token of each sequence: the same formula in another order, each within its bound."""
    for bits in (16, 8):
        lens = [1, 300, 77, 1000]
        cache, table, K, V = filled(None, lens, 32, 2, 128, BF16, bits)
        Q = normal((4, 8, 128), BF16, 3)
        a, b = torch.empty_like(Q), torch.empty_like(Q)
        cache.attend(Q, table, gpu_i32(lens), a)
        cache.attend_chunk(Q, gpu_i32([0, 1, 2, 3, 4]), table, gpu_i32(lens), b)
        _, bound = reference(Q, K, V, [1] * 4, lens, bits, 128 ** -0.5, True)
        assert_within(b, a.cpu().double(), 2 * bound, f"bits {bits}")


def test_rows_of_no_sequence_are_left_as_they_are():
    cache, table, K, V = filled(None, [100, 60], 16, 2, 64, BF16, 16)
    Q, O = normal((90, 4, 64), BF16, 1), torch.full((90, 4, 64), 7.0, dtype=BF16, device="cuda")
    cache.attend_chunk(Q, gpu_i32([0, 50, 70]), table, gpu_i32([100, 60]), O)
    ref, bound = reference(Q[:70], K, V, [50, 20], [100, 60], 16, 0.125, True)
    assert_within(O[:70], ref, bound, "rows")
    assert bool((O[70:] == 7.0).all())


def test_other_sequences_and_pages_do_not_reach_a_result():
    """NaN in one sequence's keys and values stays there; `filled` has NaN wherever nothing was written."""
    for bits in (16, 8):
        lens, new = [70, 64, 33], [20, 64, 33]
        cache, table, K, V = filled(None, lens, 32, 2, 64, BF16, bits)
        Q = normal((sum(new), 4, 64), BF16, 9)
        want, got = torch.empty_like(Q), torch.empty_like(Q)
        args = gpu_i32(offsets(new)), table, gpu_i32(lens)
        cache.attend_chunk(Q, *args, want)
        bad = torch.full((64, 2, 64), math.nan, dtype=BF16, device="cuda")
        at = torch.arange(64, device="cuda")
        cache.write(bad, bad, table[1].long()[at // 32] * 32 + at % 32)
        cache.attend_chunk(Q, *args, got)
        assert torch.equal(got[:20], want[:20]) and torch.equal(got[84:], want[84:]) and bool(got[20:84].isnan().all())


def test_lengths_beyond_the_table_are_cut():
    cache, table, K, V = filled(None, [32], 16, 1, 64, BF16, 16)
    Q = normal((5, 1, 64), BF16, 1)
    a, b, c = (torch.empty_like(Q) for _ in range(3))
    cu = gpu_i32([0, 5])
    cache.attend_chunk(Q, cu, table, gpu_i32([32]), a)
    cache.attend_chunk(Q, cu, table, gpu_i32([5000]), b)
    cache.attend_chunk(Q, cu, table, gpu_i32([-3]), c)
    assert torch.equal(a, b) and not c.any()


@pytest.mark.parametrize("bits", [16, 8])
def test_pages_beyond_32_bits(bits):
    from paper_2404_01847_amd.attention import PagedKV
    pages = 70000 if bits == 16 else 140000
    cache = PagedKV(pages, 64, 8, 64, bits=bits)
    assert cache.K.numel() * cache.K.element_size() > 1 << 32
    K, V, Q = (normal((300, 8, 64), BF16, i) for i in range(3))
    table = (pages - 1 - torch.arange(5, dtype=torch.int32, device="cuda"))[None]
    at = torch.arange(300, device="cuda")
    cache.write(K, V, table[0].long()[at // 64] * 64 + at % 64)
    small, low = PagedKV(5, 64, 8, 64, bits=bits), torch.arange(5, dtype=torch.int32, device="cuda")[None]
    small.write(K, V, at)
    outs = [c.attend_chunk(Q[:100], gpu_i32([0, 100]), t, gpu_i32([300]), torch.empty_like(Q[:100])) for c, t in ((cache, table), (small, low))]
    assert torch.equal(*outs)


@pytest.mark.parametrize("bits", [16, 8])
def test_same_bits_every_time_and_in_a_graph(bits):
    """Captured and replayed with new lengths and offsets in the same buffers, several parts and one."""
    for lens, new in (([3000], [40]), ([300, 20, 700], [100, 5, 300])):
        cache, table, K, V = filled(None, lens, 16, 2, 64, BF16, bits)
        Q, n, cu = normal((sum(new), 4, 64), BF16, 1), gpu_i32(lens), gpu_i32(offsets(new))
        O, want = torch.empty_like(Q), torch.empty_like(Q)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cache.attend_chunk(Q, cu, table, n, O)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            cache.attend_chunk(Q, cu, table, n, O)
        for cut in (0, 1, 100, 19):
            n.copy_(gpu_i32([max(0, x - cut) for x in lens]))
            Q.copy_(normal(Q.shape, BF16, cut))
            O.fill_(math.nan), want.fill_(math.nan)
            graph.replay()
            cache.attend_chunk(Q, cu, table, n, want)
            torch.cuda.synchronize()
            assert torch.equal(O, want) and O.isfinite().all()


def test_nothing_new():
    cache, table, K, V = filled(None, [32, 16], 16, 1, 64, BF16, 16)
    Q = normal((4, 1, 64), BF16, 1)
    O = torch.full_like(Q, 5.0)
    cache.attend_chunk(Q, gpu_i32([0, 0, 0]), table, gpu_i32([32, 16]), O)
    cache.attend_chunk(Q[:0], gpu_i32([0, 0, 0]), table, gpu_i32([32, 16]), O[:0])
    assert bool((O == 5.0).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_no_pages_to_see(bits):
    """A table without columns, and a cache without pages: zeros, whatever the lengths say."""
    from paper_2404_01847_amd.attention import PagedKV
    Q = normal((9, 4, 64), BF16, 1)
    for cache, table in ((PagedKV(4, 16, 2, 64, bits=bits), torch.zeros((2, 0), dtype=torch.int32, device="cuda")), (PagedKV(0, 16, 2, 64, bits=bits), torch.zeros((2, 300), dtype=torch.int32, device="cuda"))):
        O = torch.full_like(Q, math.nan)
        cache.attend_chunk(Q, gpu_i32([0, 4, 9]), table, gpu_i32([100, 5]), O)
        assert not O.any()


@pytest.mark.parametrize("bits", [16, 8])
def test_tables_offsets_and_lengths_that_hold_anything_stay_in_the_operands(bits):
    from test_gpu_attention_guards import Guarded
    import paper_2404_01847_amd as s24
    lens, page, hkv, hq, d = [400, 33, 90], 32, 2, 8, 64
    cache, table, K, V = filled(s24, lens, page, hkv, d, BF16, bits)
    Q = normal((200, hq, d), BF16, 1)
    new = Guarded()
    gen = torch.Generator().manual_seed(1)
    for cu in ([0, 100, 133, 200], [0, 1 << 30, 50, 100], [-5, 20, -7, 300], [200, 80, 70, 60]):
        for n in (lens, [1 << 30, -1, 2 ** 31 - 1], [0, 0, 5]):
            for anything in (table, torch.randint(-(1 << 31), 1 << 31, table.shape, generator=gen).to(torch.int32).cuda()):
                O = new((200, hq, d), BF16, 8)
                work = new((s24.attn_chunk_workspace(cache.buffers, table.shape[1], 200, 3, hq),), torch.uint8)
                s24.attn_chunk(cache.buffers, Q, gpu_i32(cu), anything, gpu_i32(n), O, work if work.numel() else None)
        new.check(f"{cu}")
