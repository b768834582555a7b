"""The attention half of a transformer layer, as cases that can be timed: what stands beside the sparse FFN layers in training, in
reading a prompt and in sampling.

Four kinds of case, over the widths of the workloads in s24_inputs.py and generic sizes:

  train    causal attention over packed sequences, forward and backward, on the views of one [tokens][(hq + 2 hkv) d] projection
  prompt   its forward alone; the queries of a sequence may be the last ones of more keys (a prompt read in chunks)
  decode   one new token of each sequence over a paged key-value cache of 16 or 8 bits
  cache    new tokens written to the pages (in 8 bits: quantised), and all tokens of the sequences read back as the attention takes them

Heads: hq query heads share hkv key-value heads, head h reads key-value head h // (hq // hkv).  A query i of lq sees the keys
j <= i + lk - lq.  The 8-bit cache holds, for each token and key-value head, a step s = max(max|x| / 127, 2^-126) in 32 bits and the whole
numbers nearest to x / s, ties to even.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = 64 * 128 * 8192 * 8192      # query heads x head size x queries x keys of the largest listed training case
LARGEST_CACHE = 8 * 65536 * 8 * 128   # values of the keys of the largest listed cache


def _case(name, kind, hq, hkv, d, dtype, **more):
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, **more}


def listed():
    """Lengths come from `lens_seed` between `shortest` and `longest`, or are all `longest`."""
    return [
        # workload c2's width (768 = 12 heads of 64) and tokens, as eight sequences
        _case("train_small", "train", 12, 12, 64, "bf16", seqs=8, shortest=1024, longest=1024, lens_seed=0),
        # workload c5's width (8192 = 64 heads of 128) and tokens, as one sequence; grouped heads, as layers of that width have
        _case("train_widest", "train", 64, 8, 128, "bf16", seqs=1, shortest=8192, longest=8192, lens_seed=0),
        # documents of very different lengths packed together, on a layer of width 2048
        _case("train_ragged_f16", "train", 16, 4, 128, "f16", seqs=9, shortest=1, longest=1500, lens_seed=1),
        # prompts of workload c4's width (4096 = 32 heads of 128) and tokens
        _case("prompt_wide", "prompt", 32, 32, 128, "bf16", seqs=4, shortest=4096, longest=4096, lens_seed=0, past=0),
        # the next chunks of prompts that are being read piece by piece
        _case("prompt_chunk_f16", "prompt", 64, 8, 128, "f16", seqs=3, shortest=37, longest=512, lens_seed=2, past=8000),
        # one short prompt: launch and latency
        _case("prompt_short", "prompt", 12, 12, 64, "bf16", seqs=1, shortest=17, longest=17, lens_seed=0, past=0),
        # one sequence being sampled
        _case("decode_one", "decode", 32, 32, 128, "bf16", seqs=1, shortest=1000, longest=1000, lens_seed=0, page=16, bits=16),
        # the 16 sequences that are sampled together in the FFN's case of few tokens
        _case("decode_few", "decode", 32, 32, 128, "bf16", seqs=16, shortest=1, longest=4096, lens_seed=3, page=64, bits=16),
        # long documents
        _case("decode_long_8bit", "decode", 64, 8, 128, "bf16", seqs=8, shortest=60000, longest=65536, lens_seed=4, page=256, bits=8),
        # a full server with a layer of workload c3's width (1280 = 20 heads of 64)
        _case("decode_many_8bit", "decode", 20, 20, 64, "f16", seqs=128, shortest=100, longest=4096, lens_seed=5, page=32, bits=8),
        # prompts quantised as they come, and read back for the attention of their next chunk
        _case("cache_prompt_8bit", "cache", 8, 8, 128, "bf16", seqs=4, shortest=2500, longest=4096, lens_seed=6, page=64, bits=8, past=1000),
        # a few short sequences, one new token each
        _case("cache_token", "cache", 12, 12, 64, "bf16", seqs=16, shortest=1, longest=1, lens_seed=0, page=16, bits=16, past=100),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["train", "train", "prompt", "prompt", "decode", "decode", "decode", "cache"])
    d = rng.choice([64, 128, 128, rng.choice([80, 96, 112])])
    hkv = rng.choice([1, 2, 4, 8, 8, 12, 20, 32])
    hq = hkv * rng.choice([g for g in (1, 1, 2, 4, 8) if hkv * g <= 64])
    c = _case("", kind, hq, hkv, d, rng.choice(["bf16", "bf16", "f16"]), lens_seed=rng.randrange(1 << 30))
    c.pop("name")
    if kind in ("train", "prompt"):
        longest = _log_uniform(rng, 16 if kind == "train" else 1, 8192)
        past = rng.choice([0, 0, _log_uniform(rng, 1, 8192)]) if kind == "prompt" else 0
        most = min(16384 // longest, LARGEST // (hq * d * longest * (longest + past)))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, min(most, 32))), shortest=rng.choice([1, longest, max(1, longest // 4)]))
        if kind == "prompt":
            c["past"] = past
    elif kind == "decode":
        longest = _log_uniform(rng, 1, 65536)
        most = min(256, LARGEST_CACHE // (hkv * d * longest))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, most)), shortest=rng.choice([1, longest, max(1, longest // 2)]),
                 page=rng.choice([16, 32, 64, 128, 256]), bits=rng.choice([16, 8]))
    else:
        longest = _log_uniform(rng, 1, 4096)
        past = rng.choice([0, _log_uniform(rng, 1, 4096)])
        most = min(64, LARGEST_CACHE // 16 // (hkv * d * (longest + past)))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, most)), shortest=rng.choice([1, longest]), past=past,
                 page=rng.choice([16, 32, 64, 128, 256]), bits=rng.choice([16, 8]), hq=hkv)
    return c


def _lengths(case):
    """New tokens and all tokens of each sequence.  (A part of the case and not of the seed: the work does not depend on the inputs.)"""
    rng = random.Random(case["lens_seed"])
    new = [_log_uniform(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"])]
    new[rng.randrange(len(new))] = case["longest"]
    past = case.get("past", 0)
    return new, [n + (rng.randint(past // 2, past) if past else 0) for n in new]


# ---------------------------------------------------------------------------------------------------- inputs
class _Inputs:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, shape, dtype, std=1.0):
        return (torch.randn(shape, generator=self.gen, device="cuda") * std).to(dtype)

    def keys(self, tokens, heads, d, dtype):
        """Keys have channels that are larger than others."""
        spread = torch.exp(0.5 * torch.randn((1, heads, d), generator=self.gen, device="cuda"))
        return (torch.randn((tokens, heads, d), generator=self.gen, device="cuda") * spread).to(dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.gen, device="cuda")


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _on_gpu(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _paged(case, rnd, lens):
    """Pages in no order: the table [seqs][pages of the longest], and the place of each token of all sequences, one after the other."""
    page = case["page"]
    counts = [-(-n // page) for n in lens]
    total, widest = sum(counts), max(counts)
    order = rnd.order(total)
    table = torch.zeros((len(lens), widest), dtype=torch.int32, device="cuda")
    places, first = [], 0
    for i, (n, k) in enumerate(zip(lens, counts)):
        pages = order[first:first + k]
        table[i, :k] = pages.to(torch.int32)
        at = torch.arange(n, device="cuda")
        places.append(pages[at // page] * page + at % page)
        first += k
    return total, table, torch.cat(places)


def prepare(case, seed):
    rnd, dt, kind = _Inputs(seed), DTYPES[case["dtype"]], case["kind"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    new, lens = _lengths(case)
    s = {"case": case, "new": new, "lens": lens}
    if kind in ("train", "prompt"):
        tq, tk = sum(new), sum(lens)
        if new == lens:   # views of one projection's result
            qkv = rnd.normal((tq, hq + 2 * hkv, d), dt)
            qkv[:, hq:hq + hkv] = rnd.keys(tq, hkv, d, dt)
            s["Q"], s["K"], s["V"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        else:
            s["Q"], s["K"], s["V"] = rnd.normal((tq, hq, d), dt), rnd.keys(tk, hkv, d, dt), rnd.normal((tk, hkv, d), dt)
        if kind == "train":
            s["dO"] = rnd.normal((tq, hq, d), dt, 1e-2)
        if own:
            from paper_2404_01847_amd.attention import Attention
            s["cu_q"] = _on_gpu(_offsets(new))
            s["cu_k"] = s["cu_q"] if new == lens else _on_gpu(_offsets(lens))
            s["layer"] = Attention(hq, hkv, d, tq, tk, dt)
        return s
    # the whole sequences, one after the other
    tokens = sum(lens)
    s["K"], s["V"] = rnd.keys(tokens, hkv, d, dt), rnd.normal((tokens, hkv, d), dt)
    s["pages"], s["table"], s["places"] = _paged(case, rnd, lens)
    s["cu"] = _on_gpu(_offsets(lens))
    if kind == "decode":
        s["Q"] = rnd.normal((len(lens), hq, d), dt)
        s["lengths"] = _on_gpu(lens)
        fill, written = slice(None), s["places"]
    else:   # the new ones are the last of each sequence
        is_new = torch.cat([torch.arange(n, device="cuda") >= n - k for n, k in zip(lens, new)])
        s["K_new"], s["V_new"], s["new_places"] = s["K"][is_new].contiguous(), s["V"][is_new].contiguous(), s["places"][is_new].contiguous()
        fill, written = ~is_new, s["places"][~is_new]
    if own:
        from paper_2404_01847_amd.attention import PagedKV
        s["cache"] = PagedKV(s["pages"], case["page"], hkv, d, dt, bits=case["bits"])
        s["cache"].write(s["K"][fill].contiguous(), s["V"][fill].contiguous(), written.contiguous())
        if kind == "decode":
            s["O"] = torch.empty_like(s["Q"])
        else:
            s["K_out"], s["V_out"] = torch.empty_like(s["K"]), torch.empty_like(s["V"])
        del s["K"], s["V"]
    else:
        s["cache"] = [_plain_pages(s["pages"] * case["page"], hkv, d, dt, case["bits"]) for _ in range(2)]
        for held, x in zip(s["cache"], (s["K"], s["V"])):
            _plain_write(held, x[fill], written)
        del s["K"], s["V"]
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _hidden(lq, lk, first, device):
    """Rows first .. of lq queries that are the last of lk keys: the pairs that are not visible."""
    i = torch.arange(first, lq, device=device)[:, None]
    return torch.arange(lk, device=device)[None, :] > i + (lk - lq)


def _plain_attention(q, k, v, dO, group):
    """Of one sequence: q [lq][hq][d], k and v [lk][hkv][d] in 32 bits; a few heads at a time."""
    lq, hq, d = q.shape
    lk, hkv = k.shape[:2]
    c = d ** -0.5
    O = torch.empty_like(q)
    grads = None if dO is None else (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    hidden = _hidden(lq, lk, 0, q.device)
    step = max(1, (1 << 28) // (lq * lk * group))
    for h in range(0, hkv, step):
        n = min(step, hkv - h)
        heads = slice(h * group, (h + n) * group)
        qh = q[:, heads].reshape(lq, n, group, d).permute(1, 2, 0, 3).reshape(n, group * lq, d)
        kh, vh = k[:, h:h + n].permute(1, 0, 2).contiguous(), v[:, h:h + n].permute(1, 0, 2).contiguous()
        P = torch.matmul(qh, kh.transpose(1, 2).contiguous()).mul_(c).view(n, group, lq, lk)
        P.masked_fill_(hidden, -math.inf)
        P.sub_(P.amax(dim=3, keepdim=True)).exp_()
        P.div_(P.sum(dim=3, keepdim=True))
        P = P.view(n, group * lq, lk)
        Oh = torch.matmul(P, vh)
        back = lambda x: x.view(n, group, lq, d).permute(2, 0, 1, 3).reshape(lq, n * group, d)
        O[:, heads] = back(Oh)
        if dO is not None:
            dOh = dO[:, heads].reshape(lq, n, group, d).permute(1, 2, 0, 3).reshape(n, group * lq, d)
            grads[2][:, h:h + n] = torch.matmul(P.transpose(1, 2), dOh).permute(1, 0, 2)
            dS = torch.matmul(dOh, vh.transpose(1, 2).contiguous())
            dS.sub_((dOh * Oh).sum(dim=2, keepdim=True)).mul_(P).mul_(c)
            grads[0][:, heads] = back(torch.matmul(dS, kh))
            grads[1][:, h:h + n] = torch.matmul(dS.transpose(1, 2), qh).permute(1, 0, 2)
    return O, grads


def _plain_pages(places, hkv, d, dt, bits):
    if bits == 16:
        return {"values": torch.zeros((places, hkv, d), dtype=dt, device="cuda"), "dtype": dt}
    return {"values": torch.zeros((places, hkv, d), dtype=torch.int8, device="cuda"),
            "step": torch.zeros((places, hkv, 1), dtype=torch.float32, device="cuda"), "dtype": dt}


def _plain_write(held, x, places):
    if "step" not in held:
        held["values"][places] = x
        return
    x = x.float()
    s = (x.abs().amax(dim=2, keepdim=True) / 127).clamp(min=2.0 ** -126)
    n = torch.round(x / s)
    # the quotient was rounded before it was: what is left of x, exactly, by a step in two parts of few bits
    high = (s.view(torch.int32) & -65536).view(torch.float32)
    rest = (x - n * high) - n * (s - high)
    n = n + (2 * rest > s).float() - (2 * rest < -s).float()
    held["values"][places] = n.clamp(-127, 127).to(torch.int8)
    held["step"][places] = s


def _plain_read(held, places):
    x = held["values"][places].float()
    return x * held["step"][places] if "step" in held else x


def _plain_decode(s):
    case, q = s["case"], s["Q"].float()
    n, hq, d = q.shape
    hkv, page = case["hkv"], case["page"]
    longest = max(s["lens"])
    at = torch.arange(longest, device="cuda")
    out = torch.empty_like(q)
    step = max(1, (1 << 29) // (longest * hkv * d))
    for b in range(0, n, step):
        e = min(n, b + step)
        places = s["table"][b:e].long()[:, at // page] * page + at % page
        K, V = (_plain_read(held, places).permute(0, 2, 1, 3).contiguous() for held in s["cache"])   # [n][hkv][longest][d]
        P = torch.matmul(q[b:e].view(e - b, hkv, hq // hkv, d), K.transpose(2, 3)) * d ** -0.5
        P = P.masked_fill(at >= s["lengths"][b:e, None, None, None], -math.inf)
        P = torch.exp(P - P.amax(dim=3, keepdim=True))
        out[b:e] = (torch.matmul(P, V) / P.sum(dim=3, keepdim=True)).view(e - b, hq, d)
    return out


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if own:
        if kind == "prompt":
            return s["layer"].forward(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"])
        if kind == "train":
            O = s["layer"].forward(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"])
            dQ, dK, dV = s["layer"].backward(s["Q"], s["K"], s["V"], s["dO"], s["cu_q"], s["cu_k"])
            return {"O": O, "dQ": dQ, "dK": dK, "dV": dV}
        if kind == "decode":
            return s["cache"].attend(s["Q"], s["table"], s["lengths"], s["O"])
        s["cache"].write(s["K_new"], s["V_new"], s["new_places"])
        s["cache"].read(s["table"], s["cu"], s["K_out"], s["V_out"])
        return {"K": s["K_out"], "V": s["V_out"]}
    if kind == "decode":
        return _plain_decode(s).to(dt)
    if kind == "cache":
        for held, x in zip(s["cache"], (s["K_new"], s["V_new"])):
            _plain_write(held, x, s["new_places"])
        return {name: _plain_read(held, s["places"]).to(dt) for name, held in zip("KV", s["cache"])}
    train = kind == "train"
    group = case["hq"] // case["hkv"]
    q, k, v = s["Q"].float(), s["K"].float(), s["V"].float()
    dO = s["dO"].float() if train else None
    O = torch.empty(q.shape, dtype=dt, device="cuda")
    grads = [torch.empty(x.shape, dtype=dt, device="cuda") for x in (q, k, v)] if train else None
    a, b = _offsets(s["new"]), _offsets(s["lens"])
    for i in range(len(s["new"])):
        qs, ks = slice(a[i], a[i + 1]), slice(b[i], b[i + 1])
        o, g = _plain_attention(q[qs], k[ks], v[ks], dO[qs] if train else None, group)
        O[qs] = o
        if train:
            for out, x, part in zip(grads, g, (qs, ks, ks)):
                out[part] = x
    return {"O": O, "dQ": grads[0], "dK": grads[1], "dV": grads[2]} if train else O


# ---------------------------------------------------------------------------------------------------- what it takes
def _pairs(case):
    """Visible pairs of a query and a key, of one head."""
    new, lens = _lengths(case)
    return sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, lens))


def work(case):
    """Inputs read once and outputs written once; of the causal products the visible pairs (two products forward, five backward)."""
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    new, lens = _lengths(case)
    if kind == "train":     # Q, K, V and dO in; O, dQ, dK and dV out
        return {"bytes": sum(new) * d * 2 * (4 * hq + 4 * hkv), "flops": 14.0 * _pairs(case) * hq * d}
    if kind == "prompt":
        return {"bytes": 2 * d * (2 * sum(new) * hq + 2 * sum(lens) * hkv), "flops": 4.0 * _pairs(case) * hq * d}
    held = 2 * hkv * (2 * d if case["bits"] == 16 else d + 4)   # bytes of a token in the cache
    if kind == "decode":
        return {"bytes": sum(lens) * held + 2 * len(lens) * hq * d * 2, "flops": 4.0 * sum(lens) * hq * d}
    # new tokens in and their place in the cache out; older ones from the cache; all of them out
    return {"bytes": sum(new) * 2 * hkv * d * 2 + sum(lens) * held + sum(lens) * 2 * hkv * d * 2, "flops": 0}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(q, k, v, first_key):
    """Softmax attention of the rows q [n][d], row i over the keys up to first_key + i; its weights too."""
    t = torch.mm(q, k.t()) / math.sqrt(q.shape[1])
    seen = torch.arange(k.shape[0], device=q.device)[None] <= torch.arange(q.shape[0], device=q.device)[:, None] + first_key
    t = torch.where(seen, t, torch.full_like(t, -math.inf))
    w = torch.exp(t - torch.logsumexp(t, dim=1, keepdim=True))
    return torch.mm(w, v), w


def _exact_quantised(x):
    """What the 8-bit cache holds of x [..., d], as the values it stands for."""
    s = (x.double().abs().amax(dim=-1, keepdim=True) / 127).float().clamp(min=2.0 ** -126).double()
    return torch.round(x.double() / s).clamp(-127, 127) * s


def exact(case, seed):
    global own
    if case["kind"] == "train" and case["hq"] * _pairs(case) * case["d"] > LARGEST or case["seqs"] * case["hq"] > 4096:
        return None
    kept, own = own, False
    rnd, dt, kind = _Inputs(seed), DTYPES[case["dtype"]], case["kind"]
    try:
        if kind in ("train", "prompt"):
            s = prepare(case, seed)
    finally:
        own = kept
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    new, lens = _lengths(case)
    a, b = _offsets(new), _offsets(lens)
    if kind in ("train", "prompt"):
        Q, K, V = s["Q"], s["K"], s["V"]
        O = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
        if kind == "train":
            dQ, dK, dV = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (Q, K, V))
        for i in range(len(new)):
            for h in range(hq):
                g = h * hkv // hq
                rows, cols = slice(a[i], a[i + 1]), slice(b[i], b[i + 1])
                q, k, v = Q[rows, h].double(), K[cols, g].double(), V[cols, g].double()
                o, w = _exact_rows(q, k, v, lens[i] - new[i])
                O[rows, h] = o
                if kind == "train":
                    do = s["dO"][rows, h].double()
                    dw = torch.mm(do, v.t())
                    ds = w * (dw - (w * dw).sum(dim=1, keepdim=True)) / math.sqrt(d)
                    dV[cols, g] += torch.mm(w.t(), do)
                    dQ[rows, h] = torch.mm(ds, k)
                    dK[cols, g] += torch.mm(ds.t(), q)
        return {"O": O, "dQ": dQ, "dK": dK, "dV": dV} if kind == "train" else O
    # the inputs of `prepare`, in its order
    tokens = sum(lens)
    K, V = rnd.keys(tokens, hkv, d, dt), rnd.normal((tokens, hkv, d), dt)
    _paged(case, rnd, lens)
    held = [_exact_quantised(x) if case["bits"] == 8 else x.double() for x in (K, V)]
    if kind == "cache":
        return {"K": held[0], "V": held[1]}
    Q = rnd.normal((len(lens), hq, d), dt)
    O = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    for i in range(len(lens)):
        k, v = held[0][b[i]:b[i + 1]], held[1][b[i]:b[i + 1]]
        for g in range(hkv):
            heads = slice(g * hq // hkv, (g + 1) * hq // hkv)
            t = torch.mm(Q[i, heads].double(), k[:, g].t()) / math.sqrt(d)
            O[i, heads] = torch.mm(torch.softmax(t, dim=1), v[:, g])
    return O
