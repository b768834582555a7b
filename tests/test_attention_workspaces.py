"""Which workspace a call gets, on the CPU: the library's calls are replaced by ones that note it."""
import pytest
import torch

from paper_2404_01847_amd import attention


class Calls:
    """Stands for the library: sizes as given, calls noted (their workspaces are kept, so that no two have one address by chance)."""

    def __init__(self, monkeypatch):
        self.stream, self.capturing, self.work = 1, False, []
        # looked at by the module that is tested, whatever the machine has
        monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)
        s24 = attention.s24
        monkeypatch.setattr(s24, "_stream", lambda: self.stream)
        monkeypatch.setattr(s24, "attn_decode_workspace", lambda cache, sequences, hq: 1000 * hq)
        monkeypatch.setattr(s24, "attn_fwd_workspace", lambda tq, tk, hq, hkv, d, sequences: 100 * sequences)
        monkeypatch.setattr(s24, "attn_bwd_workspace", lambda tq, tk, hq, hkv, d, sequences: 3000 - 100 * sequences)
        monkeypatch.setattr(s24, "attn_decode", lambda cache, Q, table, lengths, O, work, scale: self.note(work, O))
        monkeypatch.setattr(s24, "attn_fwd", lambda Q, K, V, O, lse, work, *a: self.note(work, O))
        monkeypatch.setattr(s24, "attn_bwd", lambda Q, K, V, O, dO, lse, dQ, dK, dV, work, *a: self.note(work, (dQ, dK, dV)))

    def note(self, work, result):
        self.work.append(work)
        return result

    def addresses(self):
        return [w.data_ptr() for w in self.work]


@pytest.fixture
def calls(monkeypatch):
    return Calls(monkeypatch)


def cache():
    return attention.PagedKV(4, 16, 2, 64, device="cpu")


def attend(c, sequences, hq=4):
    Q = torch.zeros(sequences, hq, 64, dtype=torch.bfloat16)
    return c.attend(Q, torch.zeros(sequences, 2, dtype=torch.int32), torch.zeros(sequences, dtype=torch.int32), torch.empty_like(Q))


def offsets(sequences, tokens=64):
    return torch.linspace(0, tokens, sequences + 1).to(torch.int32)


def rows(n, heads):
    return torch.zeros(n, heads, 64, dtype=torch.bfloat16)


def test_captured_calls_share_no_workspace(calls):
    """Two graphs captured on one stream, and a plain call on it: they may run at the same time."""
    c, layer = cache(), attention.Attention(4, 2, 64, 64, device="cpu")
    passes = [lambda: attend(c, 3), lambda: layer.forward(rows(64, 4), rows(64, 2), rows(64, 2), offsets(2)),
              lambda: layer.backward(rows(64, 4), rows(64, 2), rows(64, 2), rows(64, 4), offsets(2))]
    for one in passes:
        calls.work.clear()
        for capturing in (False, True, True, False):
            calls.capturing = capturing
            one()
        plain, first, second, again = calls.addresses()
        assert plain == again and len({plain, first, second}) == 3


def test_workspaces_do_not_pile_up(calls):
    """Batches of every size, of several layers and caches, over and over: what is held is the largest that a call needs."""
    caches, layers = [cache() for _ in range(3)], [attention.Attention(4, 2, 64, 64, device="cpu") for _ in range(3)]
    attention._buffers.held.clear()
    for _ in range(2):
        for n in range(1, 30):
            for c in caches:
                attend(c, n)
            for layer in layers:
                layer.forward(rows(64, 4), rows(64, 2), rows(64, 2), offsets(n))
                layer.backward(rows(64, 4), rows(64, 2), rows(64, 2), rows(64, 4), offsets(n))
    kept = list(attention._buffers.held.values())
    assert len(kept) == 1 and kept[0].numel() == 4000
    calls.work.clear()
    attend(caches[0], 5)
    layers[1].forward(rows(64, 4), rows(64, 2), rows(64, 2), offsets(3))
    assert calls.addresses() == [kept[0].data_ptr()] * 2


def test_a_larger_call_after_a_smaller_one(calls):
    attention._buffers.held.clear()
    c = cache()
    for hq in (2, 8, 4):
        attend(c, 2, hq)
    assert [w.numel() for w in calls.work] == [2000, 8000, 8000]


def test_streams_and_threads_have_their_own(calls):
    import threading
    attention._buffers.held.clear()
    c = cache()
    for calls.stream in (1, 2, 1):
        attend(c, 2)
    thread = threading.Thread(target=attend, args=(c, 2))
    thread.start()
    thread.join()
    one, two, again, other = calls.addresses()
    assert one == again and len({one, two, other}) == 3
