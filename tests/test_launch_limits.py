"""A launch holds less than 2^32 work items: of more the runtime silently runs the remainder.  Calls that would take more are refused on the host before anything is launched."""
import pytest

from test_attention_host import BF16, P, SHAPE, cache, lib, rows, shape   # noqa: F401 (lib is the fixture)
from test_rotary_host import plan

GROUPS = 1 << 24   # workgroups of 256, one too many


def test_rotation(lib):
    for tokens in (4 * GROUPS - 3, 4 * GROUPS + 5, (1 << 30) - 1):      # a wave to a token
        small = rows(1, token=16)
        assert lib.s24_rotary_fwd(plan(rotated=16), P, small, None, small, None, tokens, 1, 0, 16, BF16, None) == SHAPE
        assert lib.s24_rotary_bwd(plan(rotated=16, wq=None, wk=None), P, small, None, None, None, small, None, None, None, 0.0, tokens, 1, 0, 16, None, 0, BF16, None) == SHAPE


def test_the_cache(lib):
    one, many = rows(1, token=16), rows(16, token=2048, head=128)
    for tokens in (1 << 26, (1 << 30) - 1):
        assert lib.s24_kv_append(cache(hkv=1, d=16), plan(rotated=16), P, None, 0, one, one, None, P, tokens, BF16, None) == SHAPE
        assert lib.s24_kv_append(cache(hkv=1, d=16, pages=0), plan(rotated=16), P, None, 0, one, one, None, P, tokens, BF16, None) == SHAPE
        assert lib.s24_kv_write(cache(hkv=16, d=128), many, many, P, tokens, BF16, None) == SHAPE
        assert lib.s24_kv_read(cache(hkv=16, d=128), P, 4, P, 2, tokens, many, many, BF16, None) == SHAPE


@pytest.mark.parametrize("width", [16, 64])
def test_single_tokens(lib, width):
    """Whole sequences to a wave, and parts that another launch adds."""
    big = rows(64, token=4096)
    assert lib.s24_attn_decode(cache(hkv=64), big, 64, P, width, P, 1 << 20, 0.125, big, P, 1 << 40, BF16, None) == SHAPE


def test_packed_sequences(lib):
    big = rows(64, token=1024, head=16)
    for causal in (0, 1):
        s = dict(sequences=1, tokens_q=1 << 25, tokens_k=1 << 25, hq=64, hkv=64, d=16, causal=causal)
        assert lib.s24_attn_fwd(shape(**s), *[big] * 4, P, P, 1 << 50, BF16, None) == SHAPE
        assert lib.s24_attn_bwd(shape(**s), *[big] * 5, P, *[big] * 3, P, 1 << 50, BF16, None) == SHAPE
        s = dict(sequences=1, tokens_q=16, tokens_k=1 << 25, hq=64, hkv=64, d=16, causal=causal)      # of keys alone
        assert lib.s24_attn_bwd(shape(**s), *[big] * 5, P, *[big] * 3, P, 1 << 50, BF16, None) == SHAPE


def test_chunks(lib):
    big = rows(64, token=1024, head=16)
    assert lib.s24_attn_chunk(cache(hkv=64, d=16), big, 64, P, P, 4, P, 1, 1 << 25, 0.125, 1, big, P, 1 << 50, BF16, None) == SHAPE


def test_elementwise(lib):
    """Eight values to a work item; of bias gradients 64 features (4 of contiguous tokens) to a workgroup."""
    BF = BF16
    p, f = 1 << 15, 1 << 20                                               # p f / 8 = 2^32
    assert lib.s24_masked_decay_grad(P, P, BF, P, 1e-4, p, f, None) == SHAPE
    assert lib.s24_act_fwd(P, P, p * f, 0, BF, None) == SHAPE
    assert lib.s24_act_bwd(P, P, P, p * f, 0, BF, None) == SHAPE
    assert lib.s24_swiglu_fwd(P, P, P, p, f, 2 * f, BF, None) == SHAPE
    assert lib.s24_swiglu_bwd(P, P, P, P, P, p, f, 2 * f, BF, None) == SHAPE
    for layout in (0, 1):                                                 # both row-major, both column-major
        ld_z, ld_h = (2 * f, f) if layout == 0 else (p, p)
        assert lib.s24_glu_fwd(P, layout, ld_z, P, layout, ld_h, p, f, 0, BF, None) == SHAPE
        assert lib.s24_glu_bwd(P, layout, ld_h, P, layout, ld_z, P, p, f, 0, BF, None) == SHAPE
    n = 1 << 28
    assert lib.s24_bias_grad(P, 0, n, 8, n, P, 0.0, BF, None) == SHAPE
    assert lib.s24_bias_grad(P, 1, 8, 8, n // 4, P, 0.0, BF, None) == SHAPE
    assert lib.s24_probe_copy(P, P, 1 << 36, None) == SHAPE


def test_products(lib):
    """Of so many tokens that the tiles of 64 (16 bits: 128) of them are 2^24 workgroups of 256."""
    p = (1 << 31) - 64
    for dt in (1, 2, 0):
        assert lib.s24_dense_gemm(P, P, P, p, 64, 64, dt, None) == SHAPE
        assert lib.s24_spmm_fwd(P, P, P, P, p, 64, 64, dt, None) == SHAPE
        assert lib.s24_spmm_bwd_dx(P, P, P, P, p, 64, 64, 0.0, dt, None) == SHAPE
