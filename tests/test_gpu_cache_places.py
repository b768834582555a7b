"""Tokens written to places that do not follow each other: new tokens of many sequences, short chunks of many prompts, in batches that the kernel for many tokens takes."""
import pytest
import torch

from attention_reference import quantise

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hkv,d,dtype", [(8, 128, BF16), (5, 64, F16), (33, 80, BF16), (12, 16, BF16)])
@pytest.mark.parametrize("length", [1, 2, 3, 5, 8, 15, 17, 40])
def test_every_token_comes_to_its_place(length, hkv, d, dtype, bits):
    """Sequences of one length that start anywhere in a page, some tokens left out as padding or past the cache: the cache holds those written and what it held before."""
    from paper_2404_01847_amd.attention import PagedKV
    page, tokens = 32, 4096 if hkv < 33 else 700
    each = -(-(length + 15) // page) + 1                     # pages of a sequence
    count = -(-tokens // length)
    gen = torch.Generator().manual_seed(length + d)
    start = torch.randint(0, 16, (count,), generator=gen)
    order = torch.randperm(count, generator=gen)
    i = torch.arange(tokens)
    places = (order[i // length] * each * page + start[i // length] + i % length)
    skipped = torch.rand(tokens, generator=gen) < 0.1
    given = torch.where(skipped, torch.where(i % 2 == 0, -1 - i, count * each * page + i), places).cuda()
    K, V = (torch.randn((tokens, hkv, d), generator=gen).to(dtype) for _ in range(2))
    cache = PagedKV(count * each, page, hkv, d, dtype, bits=bits)
    for t in (cache.K, cache.V, cache.k_step, cache.v_step):
        if t is not None:
            t.fill_(3)
    cache.write(K.cuda(), V.cuda(), given)
    keep = ~skipped
    at = places[keep]
    for name, x in (("K", K), ("V", V)):
        held = getattr(cache, name).cpu()                    # a page of a head: K [page][d], V [page / E][d][E]
        if name == "V":
            E = 8 if bits == 16 else 16
            held = held.view(cache.pages, hkv, page // E, d, E).transpose(3, 4).reshape(cache.pages, hkv, page, d)
        held = held.transpose(1, 2).reshape(-1, hkv, d)
        want = torch.full_like(held, 3)
        if bits == 16:
            want[at] = x[keep]
        else:
            numbers, steps = quantise(x[keep])
            want[at] = (numbers + 128).to(torch.uint8)
            got = getattr(cache, "k_step" if name == "K" else "v_step").cpu().transpose(1, 2).reshape(-1, hkv)
            step = torch.full_like(got, 3)
            step[at] = steps[..., 0].float()
            assert torch.equal(got, step), name
        assert torch.equal(held, want), name
