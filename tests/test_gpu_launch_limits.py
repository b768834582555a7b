"""Calls as large as a launch takes, and ones beyond it (2^32 work items), which are refused."""
import math

import pytest
import torch

from attention_reference import assert_within, packed

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
SHAPE = -2


def test_rotation_of_as_many_tokens_as_a_launch_takes():
    """One head of 16: a wave to a token, 2^24 - 1 workgroups.  Four tokens more are refused, and nothing is written."""
    import paper_2404_01847_amd as s24
    most = (1 << 26) - 4
    plan = s24.RotaryPlan(16, BF16, (10000.0 ** (-torch.arange(8, dtype=torch.float64) / 8)).cuda())
    x = torch.randn((most + 4, 1, 16), dtype=BF16, device="cuda")
    at, none = torch.arange(most + 4, dtype=torch.int32, device="cuda"), x[:, :0]
    z = torch.full_like(x, math.nan)
    for forward in (True, False):
        z.fill_(math.nan)

        def call(a, b):
            if forward:
                s24.rotary_fwd(plan, x[a:b], none[a:b], at[a:b], z[a:b], none[a:b])
            else:
                s24.rotary_bwd(plan, x[a:b], none[a:b], None, None, at[a:b], z[a:b], none[a:b])
        with pytest.raises(s24.S24Error) as error:
            call(0, most + 4)
        assert error.value.status == SHAPE and bool(z.isnan().all())
        call(0, most)
        assert not bool(z[:most].isnan().any()) and bool(z[most:].isnan().all())
        for a in (0, most // 2, most - 1000):
            whole = z[a:a + 1000].clone()
            call(a, a + 1000)
            assert torch.equal(z[a:a + 1000], whole)


def test_attention_of_more_rows_than_a_launch_could_join():
    """2^28 rows of queries in whole tiles, of which none has parts that a launch of sixteen rows to a workgroup would have to add."""
    import paper_2404_01847_amd as s24
    n, count, hq, hkv, d = 1024, 4096 + 1, 64, 1, 16
    Q, dO = (torch.randn((n * count, hq, d), dtype=BF16, device="cuda") for _ in range(2))
    K, V = (torch.randn((n * count, hkv, d), dtype=BF16, device="cuda") for _ in range(2))
    O, lse = torch.full_like(Q, math.nan), torch.full((hq, n * count), math.nan, device="cuda")
    cu = torch.arange(count + 1, dtype=torch.int32, device="cuda") * n
    assert s24.attn_fwd_workspace(n * count, n * count, hq, hkv, d, count) == 0
    s24.attn_fwd(Q, K, V, O, lse, None, cu)
    work = torch.empty(s24.attn_bwd_workspace(n * count, n * count, hq, hkv, d, count), dtype=torch.uint8, device="cuda")
    grads = [torch.full_like(x, math.nan) for x in (Q, K, V)]
    s24.attn_bwd(Q, K, V, O, dO, lse, *grads, work, cu)
    assert not any(bool(x.isnan().any()) for x in (O, lse, *grads))
    for i in (0, count // 2, count - 1):
        rows = slice(i * n, (i + 1) * n)
        ref, bound = packed(Q[rows], K[rows], V[rows], [0, n], [0, n], d ** -0.5, True, dO[rows])
        for name, x in zip(("O", "dQ", "dK", "dV"), (O, *grads)):
            assert_within(x[rows], ref[name], bound[name], f"{name} of sequence {i}")


def test_a_weight_gradient_of_no_tokens_with_more_values_than_a_launch_has_work_items():
    """Cleared, all of it."""
    import paper_2404_01847_amd as s24
    q, r = 65536 + 64, 65536
    dW = torch.full((r, q), math.nan, device="cuda")
    assert dW.numel() > 1 << 32
    some = torch.empty(1024, dtype=BF16, device="cuda").data_ptr()       # (an empty tensor has no address)
    assert s24.lib().s24_dense_dw(some, some, dW.data_ptr(), 0, q, r, 0.0, s24.BF16, None) == 0
    assert not bool(dW.any())
