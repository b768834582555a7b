"""One Attention for batches of any size up to its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()


def offsets(lens):
    return torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def passes(layer, lq, lk, hq, hkv, d, seed):
    Q, K, V, dO = normal((sum(lq), hq, d), seed), normal((sum(lk), hkv, d), seed + 1), normal((sum(lk), hkv, d), seed + 2), normal((sum(lq), hq, d), seed + 3)
    cq, ck = offsets(lq), offsets(lk)
    out = [layer.forward(Q, K, V, cq, ck).clone(), layer.lse.clone()]
    return out + [x.clone() for x in layer.backward(Q, K, V, dO, cq, ck)]


@pytest.mark.parametrize("d", [64, 80])
def test_batches_up_to_the_layers_size(d):
    """What a layer of a batch's own size gives, bit for bit; also after larger and smaller ones, and with other numbers of queries than of keys."""
    from paper_2404_01847_amd.attention import Attention
    hq, hkv = 4, 2
    layer = Attention(hq, hkv, d, 300)
    for seed, (lq, lk) in enumerate((([300], [300]), ([100, 33], [100, 33]), ([1], [1]), ([20, 30], [170, 80]), ([300], [300]), ([200], [40]))):
        got = passes(layer, lq, lk, hq, hkv, d, 10 * seed)
        want = passes(Attention(hq, hkv, d, sum(lq), sum(lk)), lq, lk, hq, hkv, d, 10 * seed)
        assert all(a.shape == b.shape and torch.equal(a, b) for a, b in zip(got, want)), (lq, lk)


def test_what_does_not_fit_is_refused():
    from paper_2404_01847_amd.attention import Attention
    layer = Attention(4, 2, 64, 50, 60)
    with pytest.raises(ValueError, match="O must have shape"):
        passes(layer, [51], [51], 4, 2, 64, 0)
    with pytest.raises(ValueError, match="dK must have shape"):
        passes(layer, [50], [61], 4, 2, 64, 0)
    Q, K, dO, cu = normal((50, 4, 64), 1), normal((50, 2, 64), 2), normal((20, 4, 64), 3), offsets([20])
    layer.forward(Q, K, K, offsets([50]))
    with pytest.raises(ValueError, match="lse must have shape"):      # not the operands of the last forward pass
        layer.backward(Q[:20], K[:20], K[:20], dO, cu)


def test_decoder_layer_serves_fewer_tokens_than_it_was_made_for():
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from decoder_layer import DecoderLayer
    from paper_2404_01847_amd.attention import PagedKV
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    outs = []
    for tokens in (150, 64):
        layer = DecoderLayer(256, 512, 4, 2, 64, tokens, seed=1)
        layer.ffn.prune()
        cache, X = PagedKV(4, 64, 2, 64), normal((104, 256), 5)
        outs.append([layer.read(X[:64], [40, 24], [0, 0], cache, table), layer.read(X[64:], [10, 30], [40, 24], cache, table)])
        if tokens == 150:
            with pytest.raises(ValueError, match="150 tokens"):
                layer.step(X, X, offsets([104]))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
