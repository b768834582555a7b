"""What the attention classes and calls refuse before anything is launched, on the CPU."""
import pytest
import torch

import paper_2404_01847_amd as s24
from paper_2404_01847_amd.attention import PagedKV

SHAPE, UNSUPPORTED = -2, -6


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page,hkv,d,status", [(48, 2, 64, SHAPE), (8, 2, 64, SHAPE), (1 << 17, 1, 16, SHAPE), (16, 0, 64, SHAPE), (16, 2, 72, SHAPE), (16, 2, 0, SHAPE), (16, 2, 256, UNSUPPORTED)])
def test_a_cache_that_no_call_takes_is_refused_when_it_is_made(page, hkv, d, status, bits):
    with pytest.raises(s24.S24Error, match=f"pages of {page} tokens, {hkv} heads of {d}") as error:
        PagedKV(2, page, hkv, d, bits=bits, device="cpu")
    assert error.value.status == status


def test_caches_that_the_calls_take():
    for page, hkv, d in ((16, 1, 16), (64, 8, 128), (65536, 1, 16)):
        for bits in (16, 8):
            for dtype in (torch.bfloat16, torch.float16):
                assert PagedKV(1, page, hkv, d, dtype, bits, device="cpu").buffers.page == page
    assert PagedKV(0, 16, 2, 64, device="cpu").pages == 0
