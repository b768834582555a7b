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


def test_tensors_without_the_axes_of_an_operand_are_refused():
    """As ValueError or by the library, not as an error of what the check itself does."""
    x, cu, table, at = torch.zeros(8, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 8], dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(8, dtype=torch.int64)
    c = PagedKV(4, 16, 2, 64, device="cpu").buffers
    for scalar in (x[0, 0, 0], x[0, 0]):
        with pytest.raises(ValueError, match="K must have shape"):
            s24.kv_write(c, scalar, x, at)
        with pytest.raises(ValueError, match="K must have shape"):
            s24.kv_read(c, table, cu, scalar, x)
        with pytest.raises(ValueError, match="Q must have shape"):
            s24.attn_decode(c, scalar, table, cu[:1], x, torch.zeros(16, dtype=torch.uint8))
    for bad in (table[0, 0], table[0]):
        with pytest.raises(ValueError, match="table must have shape"):
            s24.kv_read(c, bad, cu, x, x)
        with pytest.raises(ValueError, match="table must have shape"):
            s24.attn_decode(c, x[:1], bad, cu[:1], x[:1], torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="buffers"):
        s24.KVBuffers(x[0, 0, 0], x[0, 0, 0], torch.bfloat16)
    none = x[:, :, :0]
    with pytest.raises(ValueError, match="at least one value"):
        s24.attn_fwd(none, none, none, none, None, None, cu)


def test_more_waves_than_a_launch_numbers_are_refused():
    """Windows of sixteen tokens of 65535 heads: their waves are numbered in 31 bits, whatever a launch would take."""
    from test_attention_host import BF16, OK, P, cache, rows
    write = lambda tokens: s24.lib().s24_kv_write(cache(hkv=65535, d=128), rows(65535, token=1 << 22, head=0), rows(65535, token=1 << 22, head=0), P, tokens, BF16, None)
    assert write(16 * (1 << 14) + 1) == SHAPE and write(1 << 19) == SHAPE
    assert write(0) == OK
