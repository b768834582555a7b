"""A decoder layer on libs24: attention with grouped heads and a 2:4-sparse gated FFN, in training, in reading prompts and in sampling.

    python examples/decoder_layer.py            # a training step, prompts read in chunks into an 8-bit cache, and tokens sampled after them

Y1 = X + Attention(X Wqkv^T) Wo^T,  Y = Y1 + FFN(Y1) over packed sequences; no norms and no positions, which are the caller's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2404_01847_amd as s24                                   # noqa: E402
from paper_2404_01847_amd.attention import Attention, PagedKV        # noqa: E402
from paper_2404_01847_amd.ffn import SparseFFN                       # noqa: E402


def offsets(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


class DecoderLayer:
    """Weights, buffers and call sequence of one layer: `tokens` tokens in a training step, up to as many in a call that serves."""

    def __init__(self, width, d_ff, hq, hkv, d, tokens, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        weight = lambda r, q: (torch.randn((r, q), generator=gen, device="cuda") * q ** -0.5).to(dtype)
        self.hq, self.hkv, self.d, self.tokens, self.dtype = hq, hkv, d, tokens, dtype
        self.Wqkv, self.Wo = weight((hq + 2 * hkv) * d, width), weight(width, hq * d)
        self.ffn = SparseFFN({"Wg": weight(d_ff, width), "Wu": weight(d_ff, width), "Wd": weight(width, d_ff)}, tokens, "swiglu", 2e-4, concat_gate_up=True)
        self.attention = Attention(hq, hkv, d, tokens, dtype=dtype)
        self.grads = {n: torch.empty(w.shape, dtype=torch.float32, device="cuda") for n, w in (("Wqkv", self.Wqkv), ("Wo", self.Wo))}

    def _project(self, X, W):
        return s24.dense_gemm(X, W, torch.empty((X.shape[0], W.shape[0]), dtype=self.dtype, device="cuda"))

    def _heads(self, X):
        """Q, K, V of the tokens X: views of one projection's result."""
        x = self._project(X, self.Wqkv).view(X.shape[0], self.hq + 2 * self.hkv, self.d)
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def _finish(self, X, O):
        Y1 = X + self._project(O.reshape(X.shape[0], -1), self.Wo)
        return Y1, Y1 + self.ffn.forward(Y1)[:X.shape[0]]

    # ---- training
    def step(self, X, dY, cu):
        """Forward and backward over packed sequences: Y and dX; the weights' gradients are in `grads` and in `ffn.w[...].grad`."""
        if X.shape[0] != self.tokens:   # the FFN's weight gradients go over all rows of its buffers
            raise ValueError(f"a training step of this layer takes {self.tokens} tokens, got {X.shape[0]}")
        self.ffn.prune()
        Q, K, V = self._heads(X)
        O = self.attention.forward(Q, K, V, cu)
        Y1, Y = self._finish(X, O)
        dY1 = dY + self.ffn.backward(Y1, dY)
        flat = O.reshape(X.shape[0], -1)
        s24.dense_dw(dY1, flat, self.grads["Wo"])
        dO = self._project(dY1, self.Wo.t().contiguous()).view(O.shape)
        self.attention.backward(Q, K, V, dO, cu)
        dQKV = self.attention.dQKV.view(X.shape[0], -1)
        s24.dense_dw(dQKV, X, self.grads["Wqkv"])
        return Y, dY1 + self._project(dQKV, self.Wqkv.t().contiguous())

    # ---- serving
    def read(self, X, new, past, cache, table):
        """The next `new[i]` tokens of each prompt, after the `past[i]` that the cache has: they are written to it, and attend to all."""
        every = [a + b for a, b in zip(past, new)]
        Q, K, V = self._heads(X)
        rows = torch.cat([torch.arange(a, b, device="cuda") for a, b in zip(past, every)])
        sequence = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
        cache.write(K, V, table[sequence, rows // cache.page].long() * cache.page + rows % cache.page)
        Ka, Va = (torch.empty((sum(every), self.hkv, self.d), dtype=self.dtype, device="cuda") for _ in range(2))
        cache.read(table, offsets(every), Ka, Va)
        O = self.attention.forward(Q, Ka, Va, offsets(new), offsets(every))
        return self._finish(X, O)[1]

    def sample(self, X, lengths, cache, table):
        """One new token of each sequence (X [sequences, width]); `lengths` (int32, on the device) are those with it."""
        Q, K, V = self._heads(X)
        at = lengths.long() - 1
        cache.write(K, V, table.gather(1, (at // cache.page)[:, None])[:, 0].long() * cache.page + at % cache.page)
        O = cache.attend(Q, table, lengths, torch.empty((X.shape[0], self.hq, self.d), dtype=self.dtype, device="cuda"))
        return self._finish(X, O)[1]


def main():
    width, d_ff, hq, hkv, d = 1024, 2816, 16, 4, 64
    lengths = [700, 33, 1315]
    tokens = sum(lengths)
    layer = DecoderLayer(width, d_ff, hq, hkv, d, tokens)
    X = torch.randn((tokens, width), device="cuda").to(torch.bfloat16)
    Y, dX = layer.step(X, 1e-2 * torch.randn_like(X), offsets(lengths))
    print(f"trained on {tokens} tokens of {len(lengths)} sequences: |Y| {Y.float().norm():.1f}, |dX| {dX.float().norm():.3f}, "
          f"|dWqkv| {layer.grads['Wqkv'].norm():.3f}, |dWd| {layer.ffn.w['Wd'].grad.norm():.3f}")

    # the same sequences as prompts, in two chunks, and sixteen tokens after them
    page = 64
    pages = [-(-(n + 16) // page) for n in lengths]
    cache = PagedKV(sum(pages), page, hkv, d, bits=8)
    table = torch.zeros((len(lengths), max(pages)), dtype=torch.int32, device="cuda")
    for i, n in enumerate(pages):
        table[i, :n] = torch.arange(sum(pages[:i]), sum(pages[:i + 1]))
    starts, first = offsets(lengths).tolist(), [n // 2 for n in lengths]
    part = lambda a, b: torch.cat([X[s + x:s + y] for s, x, y in zip(starts, a, b)])
    layer.read(part([0] * 3, first), first, [0] * 3, cache, table)
    rest = [n - m for n, m in zip(lengths, first)]
    out = layer.read(part(first, lengths), rest, first, cache, table)
    ends = (torch.tensor(rest).cumsum(0) - 1).tolist()
    whole = (torch.tensor(lengths).cumsum(0) - 1).tolist()
    print(f"read in two chunks: last tokens differ from the training pass by {(out[ends].float() - Y[whole].float()).norm() / Y[whole].float().norm():.4f} "
          "(the keys and values are in 8 bits)")
    now, x = torch.tensor(lengths, dtype=torch.int32, device="cuda"), out[ends]
    for _ in range(16):
        now += 1
        x = layer.sample(x * (width ** 0.5 / x.float().norm(dim=1, keepdim=True)).to(x.dtype), now, cache, table)
    torch.cuda.synchronize()
    print(f"sampled 16 tokens of {len(lengths)} sequences: lengths {now.tolist()}, |x| {x.float().norm():.1f}")


if __name__ == "__main__":
    main()
