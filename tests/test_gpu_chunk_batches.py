"""Attention of new tokens in batches that fill the device, and on both sides of 2^17 rows of all heads, where four workgroups a compute unit have whole tiles: on the GPU against 64 bits on the CPU with the bounds of
attention_reference.py (those of test_gpu_chunk.py, whose roundings are the same however a batch is cut)."""
import pytest
import torch

from test_gpu_chunk import chunk

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def spread(total, count):
    return [total // count + (i < total % count) for i in range(count)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("new,lens,causal", [([1100, 1100], [1100, 2500], True), ([2100], [2100], True), ([3, 2050, 0, 1], [900, 2300, 40, 3000], True), ([1500, 700], [800, 900], True),
                                             ([1100, 1100], [70, 1500], False), ([1200, 900], [0, 1000], True)])
def test_many_rows(new, lens, causal, dtype, bits):
    """2^17 rows of all heads and more; among them tokens that see nothing, sequences without new tokens or positions, and few rows beside many."""
    chunk(new, lens, 64, 8, 64, dtype, bits, 64, causal, seed=len(new))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [16, 48, 80, 96, 112, 128])
def test_many_rows_of_every_head_size(d, bits):
    new, lens = [2000, 97], [2000, 1000]
    chunk(new, lens, 64, 8, d, BF16, bits, 16, seed=d)


@pytest.mark.parametrize("bits", [16, 8])
def test_one_token_more(bits):
    for total in (2047, 2048):
        new, lens = [total - 60, 60], [total, 3000]
        chunk(new, lens, 64, 8, 64, BF16, bits, 64, seed=total)


@pytest.mark.parametrize("bits", [16, 8])
def test_more_tiles_than_pieces_of_a_batch_that_could_be_cut(bits):
    """Twelve sequences have more tiles than two rounds of workgroups."""
    new, lens = spread(2040, 12), [170, 400, 6000, 180, 900, 171, 1000, 200, 300, 100, 720, 2500]
    chunk(new, lens, 64, 8, 64, BF16, bits, 32, seed=12)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("total", [2047, 2300])
def test_more_sequences_than_lanes(total, bits):
    gen = torch.Generator().manual_seed(total)
    new, past = spread(total, 100), torch.randint(0, 1500, (100,), generator=gen).tolist()
    lens = [n + p for n, p in zip(new, past)]
    chunk(new, lens, 64, 8, 32, F16, bits, 64, seed=total)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("count", [260, 290])
def test_many_sequences_of_few_rows(count, bits):
    """30 rows each."""
    new, lens = [30] * count, [700 + 3 * (i % 100) for i in range(count)]
    chunk(new, lens, 16, 16, 64, BF16, bits, 64, seed=count)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new,lens,hq,hkv,d", [([600], [8000], 64, 8, 32), ([300, 41, 260], [5000, 4000, 4500], 64, 8, 80), ([1100], [9000], 32, 2, 64)])
def test_parts_of_many_rows(new, lens, hq, hkv, d, bits):
    """64 rows to a workgroup that adds parts, which is the most."""
    chunk(new, lens, hq, hkv, d, BF16, bits, 64, seed=d)
