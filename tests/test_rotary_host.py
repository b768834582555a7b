"""CPU-side checks of the rotation, of appending and of chunks: bad arguments are refused on the host before anything is launched, and nothing to do is no error."""
import ctypes as C
import math

import pytest
import torch

from test_attention_host import ALIGN, BF16, DTYPE, F32, NULL, OK, P, SHAPE, UNSUP, cache, rows

bf = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2404_01847_amd as s24
    if not os.path.exists(s24.lib_path()):
        from paper_2404_01847_amd.build import build
        build(verbose=False)
    return s24.lib()


def plan(**kw):
    from paper_2404_01847_amd.binding import _Rotary
    x = dict(frequencies=P, axis=None, wq=P, wk=P, axes=1, rotated=64, eps=1e-6, interleaved=0) | kw
    return C.byref(_Rotary(*x.values()))


def fwd(lib, r=None, at=P, tokens=4, hq=4, hkv=2, d=64, dt=BF16, **kw):
    q, k, qo, ko = (kw.get(n) or rows(4 if n in ("Q", "Qo") else 2) for n in ("Q", "K", "Qo", "Ko"))
    return lib.s24_rotary_fwd(r or plan(), at, q, k, qo, ko, tokens, hq, hkv, d, dt, None)


def bwd(lib, r=None, at=P, tokens=4, hq=4, hkv=2, d=64, dt=BF16, beta=0.0, dwq=P, dwk=P, work=P, size=1 << 40, **kw):
    x = [kw[n] if n in kw else rows(4 if n in ("Q", "Qo", "dQ") else 2) for n in ("Qo", "Ko", "Q", "K", "dQ", "dK")]
    return lib.s24_rotary_bwd(r or plan(), at, *x, dwq, dwk, beta, tokens, hq, hkv, d, work, size, dt, None)


def append(lib, c=None, r=None, at=P, hq=4, places=P, tokens=4, dt=BF16, **kw):
    q, k, v, qo = (kw.get(n) or rows(4 if n in ("Q", "Qo") else 2) for n in ("Q", "K", "V", "Qo"))
    return lib.s24_kv_append(c or cache(), r or plan(), at, q, hq, k, v, qo, places, tokens, dt, None)


def chunk(lib, c=None, hq=4, cu=P, table=P, width=4, lens=P, n=2, tokens=8, scale=0.125, causal=1, work=P, size=1 << 40, dt=BF16, **kw):
    return lib.s24_attn_chunk(c or cache(), kw.get("Q") or rows(4), hq, cu, table, width, lens, n, tokens, scale, causal, kw.get("O") or rows(4), work, size, dt, None)


def test_plans(lib):
    for call in (fwd, bwd, append):
        for bad in (dict(axes=0), dict(axes=1 << 20), dict(rotated=-16), dict(rotated=8), dict(rotated=80), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf)):
            assert call(lib, r=plan(**bad)) == SHAPE, bad
        assert call(lib, r=plan(frequencies=None)) == NULL and call(lib, at=None) == NULL
        for bad in (dict(frequencies=P + 4), dict(axis=P + 2), dict(wq=P + 8), dict(wk=P + 2)):
            assert call(lib, r=plan(**bad)) == ALIGN, bad
        assert call(lib, at=P + 2) == ALIGN and call(lib, dt=F32) == UNSUP and call(lib, dt=9) == DTYPE
        assert call(lib, tokens=-1) == SHAPE and call(lib, tokens=1 << 31) == SHAPE and call(lib, hq=-1) == SHAPE and call(lib, hq=1 << 16) == SHAPE
    assert lib.s24_rotary_fwd(None, P, None, None, None, None, 0, 0, 0, 64, BF16, None) == NULL
    for d, status in ((0, SHAPE), (72, SHAPE), (8, SHAPE), (256, UNSUP)):
        assert fwd(lib, d=d, r=plan(rotated=0)) == status and bwd(lib, d=d, r=plan(rotated=0)) == status


def test_rotary_operands(lib):
    for name in ("Q", "K", "Qo", "Ko"):
        n = 4 if name[0] == "Q" else 2
        for call in (fwd, bwd):
            assert call(lib, **{name: rows(n, data=None)}) == NULL and call(lib, **{name: rows(n, data=P + 8)}) == ALIGN and call(lib, **{name: rows(n, token=260)}) == ALIGN
            assert call(lib, **{name: rows(n, token=1 << 23)}) == SHAPE
    for bad in (dict(token=32), dict(head=32), dict(token=0)):       # rows that are written must not overlap
        assert fwd(lib, Qo=rows(4, **bad)) == SHAPE and bwd(lib, dQ=rows(4, **bad)) == SHAPE
    assert bwd(lib, Q=None) == NULL and bwd(lib, dwq=None) == NULL and bwd(lib, dwk=None) == NULL and bwd(lib, dwq=P + 2) == ALIGN
    assert bwd(lib, beta=0.5) == SHAPE and bwd(lib, beta=math.nan) == SHAPE
    assert bwd(lib, work=None) == NULL and bwd(lib, work=P + 8) == ALIGN
    need = lib.s24_rotary_bwd_workspace(plan(), 4, 4, 2, 64)
    assert need > 0 and bwd(lib, size=need - 1) == SHAPE
    assert lib.s24_rotary_bwd_workspace(plan(wq=None, wk=None), 4, 4, 2, 64) == 0 and lib.s24_rotary_bwd_workspace(None, 4, 4, 2, 64) == 0
    assert lib.s24_rotary_bwd_workspace(plan(), 1 << 20, 64, 8, 128) <= 16 << 20       # does not grow with the tokens
    # nothing to do
    assert fwd(lib, tokens=0, at=None) == OK and fwd(lib, hq=0, hkv=0) == OK
    assert bwd(lib, r=plan(wq=None, wk=None), tokens=0, Q=None, K=None, dwq=None, dwk=None, work=None, size=0) == OK
    assert lib.s24_rotary_fwd(plan(rotated=0, frequencies=None), None, None, None, None, None, 4, 0, 0, 64, BF16, None) == OK


def test_append_operands(lib):
    for bad in (dict(pages=-1), dict(page=48), dict(hkv=0), dict(d=72)):
        assert append(lib, c=cache(**bad)) == SHAPE, bad
    assert append(lib, c=cache(bits=4)) == DTYPE and append(lib, c=cache(K=None)) == NULL and append(lib, c=cache(d=256), r=plan()) == UNSUP
    assert append(lib, c=cache(d=32)) == SHAPE                           # more turned than a head has
    for name in ("Q", "K", "V", "Qo"):
        assert append(lib, **{name: rows(4 if name[0] == "Q" else 2, data=None)}) == NULL
    assert append(lib, Qo=rows(4, token=32)) == SHAPE and append(lib, K=rows(2, data=P + 8)) == ALIGN
    assert append(lib, places=None) == NULL and append(lib, places=P + 4) == ALIGN
    assert append(lib, tokens=0, places=None, at=None) == OK
    wide = rows(65535, token=1 << 22, head=0)                            # more waves than a launch numbers
    assert lib.s24_kv_append(cache(hkv=65535, d=128), plan(), P, None, 0, wide, wide, None, P, 1 << 20, BF16, None) == SHAPE


def test_chunk_operands(lib):
    for bad in (dict(pages=-1), dict(page=8), dict(hkv=0), dict(d=72)):
        assert chunk(lib, c=cache(**bad)) == SHAPE, bad
    assert chunk(lib, c=cache(bits=4)) == DTYPE and chunk(lib, dt=F32) == UNSUP and chunk(lib, c=cache(V=P + 8)) == ALIGN
    for bad in (dict(hq=3), dict(hq=0), dict(n=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(width=-1), dict(width=1 << 28), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf)):
        assert chunk(lib, **bad) == SHAPE, bad
    big = cache(hkv=1, page=65536)
    assert lib.s24_attn_chunk(big, rows(60000, token=0, head=0), 60000, P, P, 1 << 14, P, 1, 4, 0.125, 1, rows(60000, token=60000 * 64), P, 1 << 40, BF16, None) == SHAPE
    assert chunk(lib, cu=None) == NULL and chunk(lib, lens=None) == NULL and chunk(lib, table=None) == NULL
    assert chunk(lib, cu=P + 2) == ALIGN and chunk(lib, lens=P + 1) == ALIGN and chunk(lib, table=P + 2) == ALIGN and chunk(lib, work=P + 8) == ALIGN
    assert chunk(lib, Q=rows(4, token=12)) == ALIGN and chunk(lib, O=rows(4, head=32)) == SHAPE
    long = dict(width=4096, n=1)
    need = lib.s24_attn_chunk_workspace(cache(), 4096, 8, 1, 4)
    assert need > 0 and chunk(lib, **long, size=need - 1) == SHAPE and chunk(lib, **long, work=None) == NULL
    assert lib.s24_attn_chunk_workspace(cache(), 4096, 8, 1, 3) == 0 and lib.s24_attn_chunk_workspace(None, 4, 8, 1, 4) == 0
    assert chunk(lib, n=0) == OK and chunk(lib, tokens=0, cu=None, lens=None) == OK


def test_the_binding_refuses_what_the_calls_cannot_see(lib):
    """Shapes, types, strides and devices of the tensors: ValueError before the call."""
    import paper_2404_01847_amd as s24
    from paper_2404_01847_amd.attention import PagedKV, Rotary, rotary_frequencies
    f, w = rotary_frequencies(64, device="cpu"), torch.ones(64, dtype=bf)
    assert f.dtype == torch.float64 and f.shape == (32,) and f[0] == 1.0 and abs(f[-1].item() - 10000 ** (-62 / 64)) < 1e-15
    refused = lambda match, call, *a, **kw: pytest.raises(ValueError, call, *a, **kw).match(match)
    refused("frequencies must be", s24.RotaryPlan, 64, bf, f.float())
    refused("frequencies must have shape", s24.RotaryPlan, 64, bf, f.view(2, 16))
    refused("wq must have shape", s24.RotaryPlan, 64, bf, f, w[:32])
    refused("wk must be", s24.RotaryPlan, 64, bf, f, w, w.float())
    refused("axis must have shape", s24.RotaryPlan, 64, bf, f, axis=torch.zeros(16, dtype=torch.int32))
    refused("axis must be", s24.RotaryPlan, 64, bf, f, axis=torch.zeros(32, dtype=torch.int64))
    refused("bfloat16 or float16", s24.RotaryPlan, 64, torch.float32, f)
    for bad in (dict(d=32), dict(d=72), dict(eps=-1.0), dict(axes=0)):
        with pytest.raises(s24.S24Error) as error:
            s24.RotaryPlan(**(dict(d=64, dtype=bf, frequencies=f) | bad))
        assert error.value.status == SHAPE
    with pytest.raises(s24.S24Error) as error:
        s24.RotaryPlan(256, bf, f)
    assert error.value.status == UNSUP

    layer = Rotary(4, 2, 64, 8, f, w, w, axes=2, device="cpu")
    Q, K, at = torch.zeros(8, 4, 64, dtype=bf), torch.zeros(8, 2, 64, dtype=bf), torch.zeros((2, 8), dtype=torch.int32)
    refused("positions must have shape", layer.forward, Q, K, at[0])
    refused("positions must be", layer.forward, Q, K, at.long())
    refused("need positions", layer.forward, Q, K, None)
    refused("K must be", layer.forward, Q, K.half(), at)
    refused("Q and K must have shape", layer.forward, Q, K[:4], at)
    refused("Q and K must have shape", layer.forward, Q[0], K, at)
    refused("Qo must have shape", layer.forward, Q[:, :2], K, at)
    refused("Q needs unit stride", layer.forward, torch.zeros(8, 4, 128, dtype=bf)[..., ::2], K, at)
    refused("must lie on a GPU", layer.forward, Q, K, at)
    refused("dQ must have shape", layer.backward, Q[0, 0, 0], K, Q, K, at)
    work = torch.zeros(1 << 16, dtype=torch.uint8)
    backward = lambda dQ, dK, q, k, out=(Q, K): s24.rotary_bwd(layer.plan, dQ, dK, q, k, at, *out, layer.dwq, layer.dwk, 0.0, work)
    refused("Q is needed", backward, Q, K, None, K)
    refused("K must have shape", backward, Q, K, Q, K[:4])
    refused("dwq is needed", s24.rotary_bwd, layer.plan, Q, K, Q, K, at, Q, K)
    refused("dQ must have shape", backward, Q, K, Q, K, (K, K))
    refused("must lie on a GPU", backward, Q, K, Q, K)

    c, table, cu, places = PagedKV(4, 16, 2, 64, device="cpu"), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int64)
    refused("places must be", c.append, layer, Q, K, K, at, places.int())
    refused("places must have shape", c.append, layer, Q, K, K, at, places[:4])
    refused("V must have shape", c.append, layer, Q, K, Q, at, places)
    refused("positions must have shape", c.append, layer, Q, K, K, at[:1], places)
    refused("a plan for heads of 64", PagedKV(4, 16, 2, 32, device="cpu").append, layer, Q, K, K, at, places)
    refused("a plan for heads of 64", PagedKV(4, 16, 2, 64, torch.float16, device="cpu").append, layer, Q, K, K, at, places)
    refused("must lie on a GPU", c.append, layer, Q, K, K, at, places)
    attend = lambda q=Q, cu=cu, table=table, lens=cu[:2], O=Q: s24.attn_chunk(c.buffers, q, cu, table, lens, O, None)
    refused("cu must have shape", attend, cu=cu[:2])
    refused("cu must be", attend, cu=cu.long())
    refused("lengths must have shape", attend, lens=cu)
    refused("O must have shape", attend, O=K)
    refused("Q must have shape", attend, q=Q[..., :32])
    refused("table must have shape", attend, table=table[0])
    refused("must lie on a GPU", attend)
    refused("table must have shape", c.attend_chunk, Q, cu, table[0], cu[:2], Q)
    refused("Q must have shape", c.attend_chunk, Q[0], cu, table, cu[:2], Q)
    scalar = Q[0, 0, 0]
    for call in (lambda: s24.rotary_fwd(layer.plan, scalar, K, at, Q, K), lambda: s24.kv_append(c.buffers, layer.plan, scalar, K, K, at, places, Q),
                 lambda: s24.attn_chunk(c.buffers, scalar, cu, table, cu[:2], Q, None), lambda: s24.attn_chunk(c.buffers, Q, cu, table[0], cu[:2], Q, None)):
        with pytest.raises(ValueError, match="must have shape"):
            call()


def test_tensors_of_another_device_than_the_current_one_are_refused(monkeypatch):
    from paper_2404_01847_amd import binding
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 40 + device, raising=False)
    assert binding._stream_of("call", 0) == 40
    with pytest.raises(ValueError, match="device 1, the current one is 0"):
        binding._stream_of("call", 1)
    with pytest.raises(ValueError, match="must lie on a GPU"):
        binding._stream_of("call", -1)
