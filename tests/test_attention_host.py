"""CPU-side checks of the attention calls: bad arguments are refused on the host before anything is launched, and nothing to do is no error."""
import ctypes as C
import os

import pytest
import torch

OK, NULL, SHAPE, DTYPE, ALIGN, UNSUP = 0, -1, -2, -3, -4, -6
BF16, F16, F32 = 1, 2, 0
P = 0x1000  # a fake, well-aligned device address: validation never dereferences it


@pytest.fixture(scope="module")
def lib():
    import paper_2404_01847_amd as s24
    if not os.path.exists(s24.lib_path()):
        from paper_2404_01847_amd.build import build
        build(verbose=False)
    return s24.lib()


def shape(**kw):
    from paper_2404_01847_amd.binding import _AttnShape
    x = dict(cu_q=P, cu_k=P, sequences=2, tokens_q=64, tokens_k=64, hq=4, hkv=2, d=64, scale=0.125, causal=1) | kw
    return C.byref(_AttnShape(*x.values()))


def rows(heads, **kw):
    from paper_2404_01847_amd.binding import _Heads
    x = dict(data=P, token=heads * 64, head=64) | kw
    return C.byref(_Heads(*x.values()))


def cache(**kw):
    from paper_2404_01847_amd.binding import _KVCache
    x = dict(K=P, V=P, k_step=P, v_step=P, pages=8, page=16, hkv=2, d=64, bits=8) | kw
    return C.byref(_KVCache(*x.values()))


def fwd(lib, s=None, q=None, k=None, v=None, o=None, lse=P, work=P, size=1 << 40, dt=BF16):
    return lib.s24_attn_fwd(s or shape(), q or rows(4), k or rows(2), v or rows(2), o or rows(4), lse, work, size, dt, None)


def bwd(lib, s=None, lse=P, work=P, size=1 << 40, dt=BF16, **kw):
    x = [kw.get(n) or rows(4 if n in ("Q", "O", "dO", "dQ") else 2) for n in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV")]
    return lib.s24_attn_bwd(s or shape(), *x[:5], lse, *x[5:], work, size, dt, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_attention_shapes(lib, call):
    for bad in (dict(sequences=-1), dict(tokens_q=-1), dict(tokens_k=1 << 40), dict(hq=0), dict(hq=3), dict(hkv=0), dict(hkv=3), dict(d=0), dict(d=72), dict(d=8),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan"))):
        assert call(lib, shape(**bad)) == SHAPE, bad
    assert call(lib, shape(d=256)) == UNSUP and call(lib, dt=F32) == UNSUP
    assert call(lib, dt=7) == DTYPE
    assert call(lib, shape(cu_q=None)) == NULL and call(lib, shape(cu_k=None)) == NULL
    assert call(lib, shape(cu_q=P + 2)) == ALIGN
    assert call(lib, work=P + 4) == ALIGN and call(lib, lse=P + 2) == ALIGN
    assert call(lib, shape(sequences=0, tokens_q=0, tokens_k=0)) == OK          # nothing to do
    assert call(lib, shape(tokens_q=0, tokens_k=0)) == OK


def test_attention_operands(lib):
    for name in ("q", "k", "v", "o"):
        n = 4 if name in "qo" else 2
        assert fwd(lib, **{name: rows(n, data=None)}) == NULL
        assert fwd(lib, **{name: rows(n, data=P + 8)}) == ALIGN
        assert fwd(lib, **{name: rows(n, token=260)}) == ALIGN and fwd(lib, **{name: rows(n, head=68)}) == ALIGN
        assert fwd(lib, **{name: rows(n, token=-256)}) == SHAPE and fwd(lib, **{name: rows(n, token=1 << 23)}) == SHAPE
    # rows that are written must not overlap; ones that are read may
    for bad in (dict(token=32), dict(head=32), dict(token=128), dict(token=0)):
        assert fwd(lib, o=rows(4, **bad)) == SHAPE, bad
        assert bwd(lib, dQ=rows(4, **bad)) == SHAPE and bwd(lib, dK=rows(2, **(bad | ({"token": 64} if bad.get("token") == 128 else {})))) == SHAPE
    assert bwd(lib, lse=None) == NULL and bwd(lib, work=None) == NULL and bwd(lib, size=0) == SHAPE


def test_workspaces(lib):
    """Few workgroups need room for the sums of parts, many none; too little is refused."""
    assert lib.s24_attn_fwd_workspace(shape(sequences=64, tokens_q=1 << 16, tokens_k=1 << 16, hq=32, hkv=32)) == 0
    long = dict(sequences=1, tokens_q=8192, tokens_k=8192, hq=1, hkv=1)
    need = lib.s24_attn_fwd_workspace(shape(**long))
    assert need > 8192 * 64 * 4
    assert fwd(lib, shape(**long), work=P, size=need - 1) == SHAPE and fwd(lib, shape(**long), work=None) == NULL
    need = lib.s24_attn_bwd_workspace(shape(**long))
    assert need >= 8192 * 8 and bwd(lib, shape(**long), size=need - 1) == SHAPE
    assert lib.s24_attn_fwd_workspace(None) == 0 and lib.s24_attn_bwd_workspace(shape(hkv=0)) == 0
    need = lib.s24_attn_decode_workspace(cache(), 3, 4)
    assert need > 0 and lib.s24_attn_decode_workspace(cache(), 3, 5) == 0 and lib.s24_attn_decode_workspace(None, 3, 4) == 0


def test_cache_arguments(lib):
    write = lambda c=None, k=None, v=None, at=P, tokens=4, dt=BF16: lib.s24_kv_write(c or cache(), k or rows(2), v or rows(2), at, tokens, dt, None)
    read = lambda c=None, k=None, v=None, table=P, width=4, cu=P, n=2, tokens=4, dt=BF16: lib.s24_kv_read(c or cache(), table, width, cu, n, tokens, k or rows(2), v or rows(2), dt, None)
    decode = lambda c=None, q=None, o=None, hq=4, table=P, width=4, lens=P, n=2, scale=0.125, work=P, size=1 << 40, dt=BF16: lib.s24_attn_decode(
        c or cache(), q or rows(4), hq, table, width, lens, n, scale, o or rows(4), work, size, dt, None)
    for call in (write, read, decode):
        for bad in (dict(pages=-1), dict(page=8), dict(page=48), dict(page=1 << 17), dict(hkv=0), dict(d=72), dict(d=0)):
            assert call(cache(**bad)) == SHAPE, bad
        assert call(cache(bits=4)) == DTYPE and call(dt=9) == DTYPE
        assert call(cache(d=256)) == UNSUP and call(dt=F32) == UNSUP
        assert call(cache(K=None)) == NULL and call(cache(v_step=None)) == NULL
        assert call(cache(V=P + 8)) == ALIGN and call(cache(k_step=P + 4)) == ALIGN
    assert write(at=None) == NULL and write(at=P + 4) == ALIGN and write(tokens=-1) == SHAPE and write(k=rows(2, data=None)) == NULL
    assert write(tokens=0, at=None) == OK and write(cache(pages=0)) == OK
    assert read(table=None) == NULL and read(cu=None) == NULL and read(width=-1) == SHAPE and read(v=rows(2, token=32)) == SHAPE
    assert read(tokens=0) == OK and read(width=0, table=None) == OK and read(n=0) == OK
    assert decode(hq=3) == SHAPE and decode(hq=0) == SHAPE and decode(scale=0.0) == SHAPE and decode(n=-1) == SHAPE and decode(width=1 << 28) == SHAPE
    assert decode(n=1 << 20, width=1 << 12) == SHAPE                                         # more positions than 2^31
    assert decode(lens=None) == NULL and decode(work=None) == NULL and decode(table=None) == NULL and decode(lens=P + 2) == ALIGN and decode(work=P + 8) == ALIGN
    assert decode(size=lib.s24_attn_decode_workspace(cache(), 2, 4) - 1) == SHAPE
    assert decode(q=rows(4, token=12)) == ALIGN and decode(o=rows(4, head=32)) == SHAPE
    assert decode(n=0, lens=None, work=None) == OK


def test_binding_refuses_what_the_calls_cannot_see(lib):
    """Shapes, types, strides and devices of the tensors: ValueError before the call."""
    import paper_2404_01847_amd as s24
    bf, cu = torch.bfloat16, torch.tensor([0, 8], dtype=torch.int32)
    Q, K, O, lse = torch.zeros(8, 4, 64, dtype=bf), torch.zeros(8, 2, 64, dtype=bf), torch.zeros(8, 4, 64, dtype=bf), torch.zeros(4, 8)
    refused = lambda *a, match, **kw: pytest.raises(ValueError, s24.attn_fwd, *a, **kw).match(match)
    refused(Q, K, K[:4], O, lse, None, cu, match="V must have shape")
    refused(Q, K, K.half(), O, lse, None, cu, match="V must be")
    refused(Q, K, K, O.transpose(1, 2).contiguous().transpose(1, 2), lse, None, cu, match="O needs unit stride")
    refused(Q, K[:, :, :32], K, O, lse, None, cu, match="one d")
    refused(Q[0], K, K, O, lse, None, cu, match="Q and K must have shape")
    refused(Q, K, K, O, lse[:2], None, cu, match="lse must have shape")
    refused(Q, K, K, O, lse, None, cu.long(), match="cu_q must be")
    refused(Q, K, K, O, lse, None, cu[:0], match="an offset for each sequence")
    refused(Q, K, K, O, lse, None, cu, torch.zeros(3, dtype=torch.int32), match="cu_k must have shape")
    refused(Q, K, K, O, lse, None, cu, match="must lie on a GPU")
    with pytest.raises(ValueError, match="dQ must have shape"):
        s24.attn_bwd(Q, K, K, O, O, lse, K, K, K, torch.zeros(1 << 16, dtype=torch.uint8), cu)
    from paper_2404_01847_amd.attention import PagedKV
    c = PagedKV(4, 16, 2, 64, device="cpu")
    at, table = torch.zeros(8, dtype=torch.int64), torch.zeros((2, 2), dtype=torch.int32)
    for bad, match in (((K, K, at.int()), "places must be"), ((K, K, at[:4]), "places must have shape"), ((Q, K, at), "K must have shape"), ((K.half(), K.half(), at), "K must be")):
        with pytest.raises(ValueError, match=match):
            c.write(*bad)
    with pytest.raises(ValueError, match="cu must have shape"):
        c.read(table, cu, K, K)
    with pytest.raises(ValueError, match="lengths must have shape"):
        s24.attn_decode(c.buffers, Q[:2], table, cu[:1], O[:2], torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="table must have shape"):
        s24.attn_decode(c.buffers, Q[:3], table, cu, O[:3], torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="16 or 8 bits"):
        PagedKV(4, 16, 2, 64, bits=4, device="cpu")
    with pytest.raises(ValueError):
        s24.KVBuffers(torch.zeros(4, 2, 16, 64, dtype=bf), torch.zeros(4, 2, 16, 64), bf)
    with pytest.raises(ValueError):
        s24.KVBuffers(torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 64, dtype=torch.uint8), bf, torch.zeros(4, 2, 16))
