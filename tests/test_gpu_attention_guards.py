"""Nothing is written but what is the call's: every operand that a call writes lies within a larger buffer, whose other bytes have to stay as they were."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
GUARD, FILL = 1 << 16, 0xA5


class Guarded:
    """Operands with GUARD bytes on either side, and gaps between the heads' rows where `gap` says so."""

    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype, gap=0):
        size = torch.empty((), dtype=dtype).element_size()
        wide = (*shape[:-1], shape[-1] + gap)
        n = math.prod(wide) * size
        flat = torch.full((2 * GUARD + n,), FILL, dtype=torch.uint8, device="cuda")
        view = flat[GUARD:GUARD + n].view(dtype).view(wide)[..., :shape[-1]]
        mine = torch.zeros(wide, dtype=torch.bool, device="cuda")
        mine[..., :shape[-1]] = True
        self.all.append((flat, mine.view(-1, 1).expand(-1, size).reshape(-1)))
        return view

    def check(self, what):
        torch.cuda.synchronize()
        for flat, mine in self.all:
            assert bool((flat[:GUARD] == FILL).all()) and bool((flat[len(flat) - GUARD:] == FILL).all()), what
            assert bool(((flat[GUARD:len(flat) - GUARD] == FILL) | mine).all()), f"{what}: a gap"


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return [0, *torch.tensor(lens).cumsum(0).tolist()]


VALID = [([100, 33, 1], 4, 2, 64), ([3000], 1, 1, 128), ([2000], 2, 2, 80), ([700, 0, 900], 16, 4, 128), ([300] * 30, 16, 16, 96), ([17], 3, 1, 16)]


@pytest.mark.parametrize("gap", [0, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lens,hq,hkv,d", VALID)     # one part; several of the forward pass and of the gradients; a launch for each gradient; empty sequences
def test_attention_stays_in_its_operands(lens, hq, hkv, d, dtype, gap):
    import paper_2404_01847_amd as s24
    n, cu, new = sum(lens), i32(offsets(lens)), Guarded()
    Q, K, V, dO = (normal((n, h, d), dtype, i) for i, h in enumerate((hq, hkv, hkv, hq)))
    O, lse, rest = new((n, hq, d), dtype, gap), new((hq, n), torch.float32), new((n, hq, d), torch.int8)
    work = new((s24.attn_fwd_workspace(n, n, hq, hkv, d, len(lens)),), torch.uint8)
    s24.attn_fwd(Q, K, V, O, lse, work, cu, rest=rest)
    new.check("forward")
    grads = [new((n, h, d), dtype, gap) for h in (hq, hkv, hkv)]
    work = new((s24.attn_bwd_workspace(n, n, hq, hkv, d, len(lens)),), torch.uint8)
    s24.attn_bwd(Q, K, V, O, dO, lse, *grads, work, cu, rest=rest)
    new.check("backward")
    assert all(x.isfinite().all() for x in (O, lse, *grads))


@pytest.mark.parametrize("bad", [[0, 1 << 30, 50, 100], [-5, 20, -7, 300], [90, 80, 70, 60], [0, 100, 100, 2 ** 31 - 1]])
def test_attention_stays_in_its_operands_whatever_the_offsets(bad):
    import paper_2404_01847_amd as s24
    n, hq, hkv, d, new = 100, 2, 1, 64, Guarded()
    Q, K, V = normal((n, hq, d), BF16, 1), normal((n, hkv, d), BF16, 2), normal((n, hkv, d), BF16, 3)
    for cq, ck in ((bad, bad), (bad, [0, 30, 60, 100]), ([0, 30, 60, 100], bad)):
        O, lse, rest = new((n, hq, d), BF16, 8), new((hq, n), torch.float32), new((n, hq, d), torch.int8)
        grads = [new((n, h, d), BF16, 8) for h in (hq, hkv, hkv)]
        O.zero_(), lse.zero_(), rest.zero_()
        s24.attn_fwd(Q, K, V, O, lse, new((s24.attn_fwd_workspace(n, n, hq, hkv, d, 3),), torch.uint8), i32(cq), i32(ck), rest=rest)
        s24.attn_bwd(Q, K, V, O, Q, lse, *grads, new((s24.attn_bwd_workspace(n, n, hq, hkv, d, 3),), torch.uint8), i32(cq), i32(ck), rest=rest)
        new.check(f"{cq} {ck}")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lens,hq,hkv,d,page", [([20000, 1, 300], 8, 2, 128, 64), ([0, 70, 128], 12, 12, 64, 16), ([500] * 70, 4, 1, 80, 32), ([40] * 300, 3, 3, 112, 16)])
def test_the_cache_stays_in_its_operands(lens, hq, hkv, d, page, bits):
    """Written in one call and token by token, read back, attended over in shares and by whole sequences; then with places, tables, offsets and lengths that hold anything."""
    import paper_2404_01847_amd as s24
    counts = [-(-x // page) for x in lens]
    pages, n, new = sum(counts), sum(lens), Guarded()
    held = [new((pages, hkv, page, d), torch.uint8 if bits == 8 else BF16) for _ in range(2)]
    steps = [new((pages, hkv, page), torch.float32) for _ in range(2)] if bits == 8 else []
    cache = s24.KVBuffers(*held, BF16, *steps)
    table, places, at = torch.zeros((len(lens), max(counts)), dtype=torch.int32), [], 0
    for i, (x, k) in enumerate(zip(lens, counts)):
        table[i, :k] = torch.arange(at, at + k)
        places.append(torch.arange(x) + at * page)
        at += k
    places, table = torch.cat(places).cuda(), table.cuda()
    K, V = normal((n, hkv, d), BF16, 1), normal((n, hkv, d), BF16, 2)
    s24.kv_write(cache, K, V, places)
    for i in range(0, min(n, 90), 30):
        s24.kv_write(cache, K[i:i + 30], V[i:i + 30], places[i:i + 30])
    new.check("written")
    Ko, Vo = (new((n, hkv, d), BF16, 8) for _ in range(2))
    s24.kv_read(cache, table, i32(offsets(lens)), Ko, Vo)
    new.check("read")
    assert torch.equal(Ko, K) and torch.equal(Vo, V) if bits == 16 else bool(Ko.isfinite().all())
    Q, O = normal((len(lens), hq, d), BF16, 3), new((len(lens), hq, d), BF16, 8)
    work = new((s24.attn_decode_workspace(cache, len(lens), hq),), torch.uint8)
    s24.attn_decode(cache, Q, table, i32(lens), O, work)
    new.check("attended")
    assert O.isfinite().all()
    gen = torch.Generator().manual_seed(4)
    s24.kv_write(cache, K, V, torch.randint(-(1 << 40), 1 << 40, (n,), generator=gen).cuda())
    s24.kv_write(cache, K, V, torch.arange(n, device="cuda") + pages * page - 100)
    anything = torch.randint(-(1 << 31), 1 << 31, table.shape, generator=gen).to(torch.int32).cuda()
    s24.kv_read(cache, anything, i32([-4, *[3 * n] * len(lens)]), Ko, Vo)
    s24.attn_decode(cache, Q, anything, i32([1 << 30] * len(lens)), O, work)
    new.check("anything")
