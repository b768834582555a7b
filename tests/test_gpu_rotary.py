"""Norms and rotations of heads, and what is appended to the cache with them, on the GPU against 64 bits on the CPU (rotary_reference.py, which derives the bounds)."""
import math

import pytest
import torch

import rotary_reference as reference
from attention_reference import assert_within

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def s24():
    import paper_2404_01847_amd as s24
    return s24


def normal(shape, dtype, seed, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(dtype).cuda()


def frequencies(rotated, base=10000.0):
    return base ** (torch.arange(rotated // 2, dtype=torch.float64) * (-2.0 / max(rotated, 1)))


class Case:
    """Operands of one call: a layer, Q, K (views of a projection, of [heads][tokens][d] buffers, or whole), gradients, positions; and results in 64 bits."""

    def __init__(self, tokens, hq, hkv, d, dtype, rotated=None, norms=(True, True), axes=1, interleaved=False, views="projection", seed=0, eps=1e-6, far=0, axis=None):
        from paper_2404_01847_amd.attention import Rotary
        rotated = d if rotated is None else rotated
        self.what = f"{tokens} tokens, heads {hq}/{hkv} of {d}, {rotated} turned, {dtype} norms {norms} axes {axes} interleaved {interleaved} {views}"
        self.shape = tokens, hq, hkv, d
        self.dtype, self.eps, self.rotated, self.interleaved = dtype, eps, rotated, interleaved
        if views == "projection":
            x, g = normal((tokens, hq + 2 * hkv, d), dtype, seed), normal((tokens, hq + 2 * hkv, d), dtype, seed + 1, 1e-2)
            part = lambda t: (t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:])
        elif views == "heads":
            x, g = normal((hq + 2 * hkv, tokens, d), dtype, seed), normal((hq + 2 * hkv, tokens, d), dtype, seed + 1, 1e-2)
            part = lambda t: tuple(v.transpose(0, 1) for v in (t[:hq], t[hq:hq + hkv], t[hq + hkv:]))
        else:
            x, g = normal((tokens, hq + 2 * hkv, d), dtype, seed), normal((tokens, hq + 2 * hkv, d), dtype, seed + 1, 1e-2)
            part = lambda t: tuple(v.contiguous() for v in (t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:]))
        self.Q, self.K, self.V = part(x)
        self.dQ, self.dK, _ = part(g)
        self.w = [normal((d,), dtype, seed + 2 + i, 0.3, 1.0) if n else None for i, n in enumerate(norms)]
        gen = torch.Generator().manual_seed(seed + 5)
        self.positions = (torch.randint(-50, 3000, (axes, tokens), generator=gen) + far).to(torch.int32).cuda()
        f = frequencies(rotated)
        if axis is None and axes > 1:
            axis = torch.randint(0, axes, (rotated // 2,), generator=gen).to(torch.int32)
        self.axis = axis
        self.layer = Rotary(hq, hkv, d, tokens, f.cuda() if rotated else None, *self.w, eps=eps, axis=None if axis is None else axis.cuda(), axes=axes, interleaved=interleaved, dtype=dtype)
        self.angle = reference.angles(self.positions, f, axis)
        self.at = dict(eps=eps, angle=self.angle, rotated=rotated, interleaved=interleaved)

    def forward(self, i):
        return reference.forward((self.Q, self.K)[i], self.w[i], **self.at)

    def check_forward(self, got, names="QK"):
        for i, name in enumerate("QK"):
            if name in names:
                ref, bound = self.forward(i)
                assert_within(got[i], ref, reference.rounded(ref, bound, self.dtype), f"{name}, {self.what}")

    def check(self):
        got = self.layer.forward(self.Q, self.K, self.positions)
        self.check_forward(got)
        out = tuple(torch.full_like(x, math.nan) for x in (self.dQ, self.dK))
        self.layer.backward(self.dQ, self.dK, self.Q, self.K, self.positions, out=out)
        for i, (name, w, dw) in enumerate(zip("QK", self.w, (self.layer.dwq, self.layer.dwk))):
            dx, ref, bound, of_dw = reference.backward((self.dQ, self.dK)[i], (self.Q, self.K)[i], w, **self.at)
            assert_within(out[i], dx, reference.rounded(dx, bound, self.dtype), f"d{name}, {self.what}")
            if w is not None:
                assert_within(dw, ref, of_dw, f"dw{name}, {self.what}")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens", [1, 2, 3, 17, 64, 65, 300])
def test_tokens(tokens, d, dtype):
    Case(tokens, 4, 2, d, dtype).check()


def test_more_rows_than_the_workgroups_take_in_one_go():
    Case(16000, 64, 8, 16, BF16).check()


@pytest.mark.parametrize("norms", [(True, True), (False, False), (True, False), (False, True)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (8, 8), (12, 4), (64, 8), (17, 16), (5, 0), (0, 3)])
def test_heads(hq, hkv, norms):
    Case(21, hq, hkv, 128, BF16, norms=norms, seed=hq).check()
    Case(21, hq, hkv, 64, F16, norms=norms, seed=hq).check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 112, 128])
def test_head_sizes_and_how_many_values_are_turned(d, dtype, interleaved):
    for rotated in sorted({0, 16, d // 32 * 16, d}):
        for norm in (True, False):
            Case(9, 6, 3, d, dtype, rotated, (norm, norm), interleaved=interleaved, seed=d + rotated).check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes", [2, 3, 5])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_several_axes(d, axes, interleaved):
    Case(50, 6, 2, d, BF16, axes=axes, interleaved=interleaved, seed=axes).check()
    Case(50, 6, 2, d, F16, d // 32 * 16, (False, False), axes=axes, interleaved=interleaved, seed=axes).check()


def test_an_axis_that_a_token_does_not_have_is_the_last_one():
    axis = torch.tensor([0, 1, 2, 3, -1, 1 << 30, -(1 << 31), 2 ** 31 - 1], dtype=torch.int32)
    Case(30, 2, 1, 16, BF16, axes=3, axis=axis).check()


def test_several_axes_without_a_choice_turn_by_the_first(s24):
    a, b = (Case(30, 2, 1, 64, BF16, axes=n, axis=None if n == 1 else torch.zeros(32, dtype=torch.int32), seed=2) for n in (1, 3))
    b.positions[0] = a.positions[0]
    plan = s24.RotaryPlan(64, BF16, frequencies(64).cuda(), *b.w, axes=3)
    Q, K = s24.rotary_fwd(plan, b.Q, b.K, b.positions, torch.empty_like(b.Q), torch.empty_like(b.K))
    for x, y in zip((Q, K), a.layer.forward(a.Q, a.K, a.positions[0])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("views", ["projection", "heads", "whole"])
def test_strides(views):
    Case(33, 6, 2, 128, BF16, views=views).check()
    Case(33, 6, 2, 64, F16, views=views, norms=(False, False)).check()


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 4000, -(1 << 31) + 50])
def test_far_positions_turn_as_exactly_as_near_ones(far):
    """fp64 angles of the reference are off by 2^-53 of up to 2^31 radians, 2^-22, which the bound has room for."""
    Case(40, 4, 2, 128, F16, norms=(False, False), far=far).check()
    Case(40, 4, 2, 64, BF16, axes=2, far=far).check()


def test_frequencies_of_any_size():
    """Whole turns a step, half turns, none, more than one, negative ones."""
    from paper_2404_01847_amd.attention import Rotary
    f = torch.tensor([0.0, math.pi, 2 * math.pi, 1e-12, 100.0, -1.0, -1e-3, 12345.678], dtype=torch.float64)
    at = torch.tensor([[0, 1, -1, 2, 3, 1000, 65537]], dtype=torch.int32).cuda()
    Q = normal((7, 2, 16), F16, 1)
    layer = Rotary(2, 0, 16, 7, f.cuda(), dtype=F16)
    z, _ = layer.forward(Q, Q[:, :0], at)
    angle = reference.angles(at, f, None)
    ref, bound = reference.forward(Q, None, 0.0, angle, 16, False)
    # 12345.678 radians a step: the angle in 64 bits and the fraction of a turn are each off by 2^-53 of up to 2^13.6 * 2^16
    assert_within(z, ref, reference.rounded(ref, bound + 2.0 ** -21 * Q.cpu().double().abs().amax(2, keepdim=True), F16), "frequencies")


@pytest.mark.parametrize("d,norm", [(128, False), (64, False), (128, True), (80, True)])
def test_in_place(s24, d, norm):
    """Gradients over those that come in, and without norms the results over the operands, have the bits of separate buffers."""
    c = Case(77, 6, 2, d, BF16, norms=(norm, norm))
    want = [x.clone() for x in c.layer.forward(c.Q, c.K, c.positions)]
    separate = c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=(torch.empty_like(c.dQ), torch.empty_like(c.dK)))
    own = c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions)
    assert own[0] is c.dQ and all(torch.equal(a, b) for a, b in zip(separate, own))
    got = c.layer.forward(c.Q, c.K, c.positions, out=(c.Q, c.K))
    assert got[0] is c.Q and all(torch.equal(a, b) for a, b in zip(got, want))


def test_weight_gradients_are_added_and_repeat(s24):
    c = Case(500, 12, 4, 64, BF16, seed=3)
    run = lambda beta: c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=(torch.empty_like(c.dQ), torch.empty_like(c.dK)), beta=beta)
    run(0.0)
    first = c.layer.dwq.clone(), c.layer.dwk.clone()
    c.layer.dwq.fill_(math.nan)
    run(0.0)
    assert torch.equal(c.layer.dwq, first[0]) and torch.equal(c.layer.dwk, first[1])      # what it held is not read
    run(1.0)
    assert torch.equal(c.layer.dwq, first[0] * 2) and torch.equal(c.layer.dwk, first[1] * 2)


def test_no_tokens(s24):
    c = Case(0, 4, 2, 64, BF16)
    c.layer.dwq.fill_(3.0), c.layer.dwk.fill_(4.0)
    c.layer.forward(c.Q, c.K, c.positions)
    c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, beta=1.0)
    assert bool((c.layer.dwq == 3.0).all()) and bool((c.layer.dwk == 4.0).all())
    c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions)
    assert not c.layer.dwq.any() and not c.layer.dwk.any()


@pytest.mark.parametrize("hq,hkv", [(0, 3), (5, 0), (0, 0)])
def test_weights_of_no_heads_have_the_gradient_zero(s24, hq, hkv):
    for norms in ((True, True), (True, False), (False, True)):
        c = Case(50, hq, hkv, 64, BF16, norms=norms)
        for beta, want in ((1.0, 3.0), (0.0, 0.0)):
            for x in (c.layer.dwq, c.layer.dwk):
                if x is not None:
                    x.fill_(3.0)
            c.layer.backward(c.dQ.clone(), c.dK.clone(), c.Q, c.K, c.positions, beta=beta)
            for x, heads in ((c.layer.dwq, hq), (c.layer.dwk, hkv)):
                assert x is None or heads > 0 or bool((x == want).all())


def test_fewer_tokens_than_the_layer_has(s24):
    c = Case(100, 6, 2, 128, BF16)
    want = [x.clone() for x in c.layer.forward(c.Q, c.K, c.positions)]
    for n in (1, 37, 99):
        got = c.layer.forward(c.Q[:n], c.K[:n], c.positions[:, :n].contiguous())
        assert all(torch.equal(a, b[:n]) for a, b in zip(got, want))
    with pytest.raises(ValueError, match="Qo must have shape"):
        more = torch.cat([c.Q, c.Q])
        c.layer.forward(more, torch.cat([c.K, c.K]), torch.cat([c.positions, c.positions], 1))


def test_gradients_against_differences(s24):
    """The gradient's product with a direction against the difference of the forward formula in 64 bits along it, which is off by the third derivative: (1e-4)^2."""
    c = Case(6, 4, 2, 64, F16, 32, eps=1e-3, axes=2)
    out = c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=(torch.empty_like(c.dQ), torch.empty_like(c.dK)))
    for i, dw in enumerate((c.layer.dwq, c.layer.dwk)):
        x, w, dz = (c.Q, c.K)[i].cpu().double(), c.w[i].cpu().double(), (c.dQ, c.dK)[i].cpu().double()
        loss = lambda x, w: (reference.forward(x, w, **c.at)[0] * dz).sum().item()
        for seed in range(4):
            gen = torch.Generator().manual_seed(seed)
            along, of_w = torch.randn(x.shape, generator=gen, dtype=torch.float64), torch.randn(w.shape, generator=gen, dtype=torch.float64)
            step = 1e-4
            for direction, got, moved in ((along, out[i], lambda t: loss(x + t * along, w)), (of_w, dw, lambda t: loss(x, w + t * of_w))):
                slope = (moved(step) - moved(-step)) / (2 * step)
                terms = got.cpu().double() * direction
                assert abs(terms.sum().item() - slope) <= 2.0 ** -10 * terms.abs().sum().item() + 1e-6


def test_what_is_no_number_stays_in_its_head(s24):
    for norm in (True, False):
        c = Case(10, 6, 2, 128, BF16, norms=(norm, norm))
        c.Q[3, 2, 17], c.K[5, 1, 100] = math.nan, math.inf
        z, k = c.layer.forward(c.Q, c.K, c.positions)
        assert z[3, 2].isnan().any() and z.isnan().any(2).nonzero().tolist() == [[3, 2]]
        assert (~k[5, 1].isfinite()).any() and (~k.isfinite()).any(2).nonzero().tolist() == [[5, 1]]


def test_values_that_are_not_turned_are_left_as_they_are():
    c = Case(10, 3, 3, 96, F16, 32, (False, False))
    c.Q[1, 1, 50:60] = math.inf
    z, k = c.layer.forward(c.Q, c.K, c.positions)
    assert torch.equal(z[..., 32:], c.Q[..., 32:]) and torch.equal(k[..., 32:], c.K[..., 32:]) and z[..., :32].isfinite().all()


def test_small_and_large_heads(s24):
    """eps decides for small ones; squares of large ones stay within fp32."""
    for std in (1e-6, 1e-3, 300.0):
        c = Case(20, 4, 2, 128, BF16, seed=9)
        c.Q.mul_(std), c.K.mul_(std)
        c.check()
    c = Case(4, 2, 1, 64, BF16, eps=1e-6)
    c.Q.zero_()
    assert not c.layer.forward(c.Q, c.K, c.positions)[0].any()


def test_in_a_graph_beside_plain_calls(s24):
    """Forward and backward captured together, replayed with new values and positions; the layer's plain calls between."""
    c = Case(200, 8, 2, 128, BF16)
    outs = tuple(torch.empty_like(x) for x in (c.dQ, c.dK))
    def both():
        c.layer.forward(c.Q, c.K, c.positions)
        c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=outs)
    results = lambda: [x.clone() for x in (c.layer.Q, c.layer.K, *outs, c.layer.dwq, c.layer.dwk)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for seed in range(4):
        c.Q.copy_(normal(c.Q.shape, BF16, seed)), c.dQ.copy_(normal(c.dQ.shape, BF16, seed + 9))
        c.positions.add_(17)
        both()
        want = results()
        for x in (c.layer.Q, c.layer.K, *outs, c.layer.dwq, c.layer.dwk):
            x.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(), want))


# ---------------------------------------------------------------------------------------------------- appending
def scattered(tokens, page, seed, spare=2):
    """Places of the tokens, in runs of different lengths in pages of any order, and the pages that a cache needs for them."""
    gen = torch.Generator().manual_seed(seed)
    pages = -(-tokens // page) + spare
    at = torch.randperm(pages, generator=gen).repeat_interleave(page) * page + torch.arange(page).repeat(pages)
    skip = int(torch.randint(0, page, (1,), generator=gen))
    return at[skip:skip + tokens].cuda(), pages


def same(a, b, names=("K", "V", "k_step", "v_step")):
    return all(torch.equal(getattr(a, n).view(torch.uint8), getattr(b, n).view(torch.uint8)) for n in names if getattr(a, n) is not None)


def empty_cache(pages, page, hkv, d, dtype, bits):
    from paper_2404_01847_amd.attention import PagedKV
    cache = PagedKV(pages, page, hkv, d, dtype, bits)
    for x in (cache.K, cache.V, cache.k_step, cache.v_step):
        if x is not None:
            x.zero_()
    return cache


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,hq,hkv,d,page", [(1, 4, 2, 64, 16), (3, 64, 8, 128, 32), (40, 12, 12, 64, 16), (1500, 16, 8, 128, 64), (2000, 6, 6, 64, 16), (1700, 8, 8, 80, 32), (30, 5, 5, 48, 16),
                                                  (900, 0, 16, 112, 128)])
def test_sixteen_bits_hold_what_the_two_calls_leave(tokens, hq, hkv, d, page, dtype, norm):
    c = Case(tokens, hq, hkv, d, dtype, norms=(norm, norm), axes=2, seed=tokens)
    places, pages = scattered(tokens, page, tokens)
    places[tokens // 2] = -1
    places[tokens // 3] = pages * page + 5
    one, two = (empty_cache(pages, page, hkv, d, dtype, 16) for _ in range(2))
    Q, K = c.layer.forward(c.Q, c.K, c.positions)
    two.write(K, c.V, places)
    got = one.append(c.layer, c.Q, c.K, c.V, c.positions, places, out=torch.full_like(c.Q, math.nan))
    assert torch.equal(got, Q) and same(one, two)
    c.check_forward((Q, K))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,hq,hkv,d,page", [(1, 4, 2, 64, 16), (40, 12, 12, 64, 16), (1500, 16, 8, 128, 64), (2000, 6, 6, 64, 16), (300, 4, 2, 80, 32), (30, 5, 5, 48, 16), (33, 2, 2, 16, 16)])
def test_eight_bits_hold_what_is_nearest(tokens, hq, hkv, d, page, dtype):
    """Of K: the step is that of the exact values up to their fp32 error, and what is held lies within half a step of them (and that error); V as the cache's write leaves it."""
    c = Case(tokens, hq, hkv, d, dtype, seed=tokens, interleaved=tokens % 2 == 0)
    places, pages = scattered(tokens, page, tokens)
    one, two = (empty_cache(pages, page, hkv, d, dtype, 8) for _ in range(2))
    two.write(c.K, c.V, places)
    got = one.append(c.layer, c.Q, c.K, c.V, c.positions, places)
    c.check_forward((got, None), "Q")
    assert same(one, two, ("V", "v_step"))
    z, bound = c.forward(1)
    at = places.cpu()
    step = one.k_step.cpu().double()[at // page, :, at % page]
    held = (one.K.cpu().double()[at // page, :, at % page] - 128) * step[..., None]
    most = z.abs().amax(2)
    assert bool(((step - most / 127).abs() <= bound.amax(2) / 127 + 2.0 ** -23 * step).all())
    assert bool(((held - z).abs() <= 0.5 * step[..., None] * (1 + 2.0 ** -14) + bound).all())
    written = torch.zeros(pages * page, dtype=torch.bool)
    written[at] = True
    assert not one.K.transpose(1, 2).reshape(pages * page, -1)[~written.cuda()].any()


@pytest.mark.parametrize("bits", [16, 8])
def test_append_over_the_queries_themselves(bits):
    c = Case(60, 8, 2, 128, BF16)
    places, pages = scattered(60, 16, 1)
    cache = empty_cache(pages, 16, 2, 128, BF16, bits)
    want = cache.append(c.layer, c.Q, c.K, c.V, c.positions, places).clone()
    assert cache.append(c.layer, c.Q, c.K, c.V, c.positions, places, out=c.Q) is c.Q and torch.equal(c.Q, want)


def test_appended_zeros_and_what_is_no_number():
    """Zeros have the smallest step; a key that holds NaN or an infinity has the step NaN, and no other."""
    c = Case(40, 2, 2, 64, BF16, norms=(False, False))
    c.K[3] = 0.0
    c.K[7, 1, 5], c.K[9, 0, 40] = math.nan, math.inf
    cache = empty_cache(3, 16, 2, 64, BF16, 8)
    cache.append(c.layer, c.Q, c.K, c.V, c.positions, torch.arange(40, device="cuda"))
    steps = cache.k_step.transpose(1, 2).reshape(48, 2)[:40]
    assert bool((steps[3] == 2.0 ** -126).all()) and steps.isnan().nonzero().tolist() == [[7, 1], [9, 0]]
    assert bool((cache.K.transpose(1, 2).reshape(48, 2, 64)[3] == 128).all())


def test_append_in_a_graph():
    """A token of each of 20 sequences, captured and replayed with new values, positions and places."""
    c = Case(20, 8, 4, 128, BF16)
    one, two = (empty_cache(30, 16, 4, 128, BF16, 8) for _ in range(2))
    places = torch.arange(20, device="cuda") * 16
    out = torch.empty_like(c.Q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one.append(c.layer, c.Q, c.K, c.V, c.positions, places, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one.append(c.layer, c.Q, c.K, c.V, c.positions, places, out=out)
    two.append(c.layer, c.Q, c.K, c.V, c.positions, places)
    for seed in range(4):
        c.Q.copy_(normal(c.Q.shape, BF16, seed)), c.K.copy_(normal(c.K.shape, BF16, seed + 5)), c.V.copy_(normal(c.V.shape, BF16, seed + 10))
        c.positions.add_(1), places.add_(1)
        graph.replay()
        want = two.append(c.layer, c.Q, c.K, c.V, c.positions, places)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and same(one, two)
