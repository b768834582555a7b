"""What stands between a layer's projection and its attention, and the attention of new tokens over what was written: norms of queries and keys for each
head with the rotation of their positions, keys and values appended to a paged cache on the way, and chunks of new tokens attending over it.

Three kinds of case, over the widths of the workloads in s24_inputs.py and generic sizes:

  rotary   training: queries and keys normalised and rotated, and the gradients of both (of the norms' weights too)
  append   serving: new tokens' queries rotated, their keys rotated and their values as they are written to pages of 16 or 8 bits; the sequences are
           read back, as what the cache holds
  chunk    serving: the last tokens of each sequence attend to all of its positions in a paged cache of 16 or 8 bits

A head x of d values is normalised to y_i = x_i w_i / sqrt(mean(x^2) + eps) (or taken as it is), and its first `rotated` values are turned in pairs p by the
angle position * frequency_p: pairs are (p, p + rotated / 2), or (2p, 2p + 1) where `interleaved`.  A token has one position, or one for each of several axes
(time, height, width), of which a pair turns by one.  Heads: hq query heads share hkv key-value heads.  Query i of lq sees the keys j <= i + lk - lq.  The 8-bit cache holds, for
each token and key-value head, a step s = max(max|x| / 127, 2^-126) in 32 bits and the whole numbers nearest to x / s.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
LARGEST_ROWS = 72 * 128 * 8192                        # values of queries and keys of the largest listed training case
LARGEST_SCORES = 64 * 128 * 4 * 1024 * 24000          # query heads x head size x queries x keys, about, of the largest listed chunk
LARGEST_CACHE = 4 * 32768 * 8 * 128                   # values of the keys of its cache


def _case(name, kind, hq, hkv, d, dtype, **more):
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, **more}


def _turn(norm, axes, rotated, interleaved=False, base=10000.0, start=0):
    return {"norm": norm, "axes": axes, "rotated": rotated, "interleaved": interleaved, "base": base, "start": start}


def listed():
    """Lengths come from `lens_seed` between `shortest` and `longest`, or are all `longest`."""
    return [
        # workload c5's width (8192 = 64 heads of 128) and tokens, grouped heads, with norms: a training step of the widest layer
        _case("norms_widest", "rotary", 64, 8, 128, "bf16", seqs=1, shortest=8192, longest=8192, lens_seed=0, **_turn(True, 1, 128, base=500000.0)),
        # workload c2's width (768 = 12 heads of 64) and tokens: the rotation alone, neighbouring values as pairs
        _case("rotation_f16", "rotary", 12, 12, 64, "f16", seqs=8, shortest=1024, longest=1024, lens_seed=0, **_turn(False, 1, 64, True)),
        # text and video of very different lengths packed together: time, height and width, with norms
        _case("video_train", "rotary", 16, 4, 128, "bf16", seqs=9, shortest=1, longest=1500, lens_seed=1, **_turn(True, 3, 128, base=1000000.0)),
        # one image's patches, height and width: few tokens of heads that are no power of two
        _case("image_train_f16", "rotary", 16, 16, 80, "f16", seqs=1, shortest=729, longest=729, lens_seed=0, **_turn(False, 2, 80)),
        # one new token of each of 16 sequences that are sampled together, far into long documents: launch and latency
        _case("append_tokens", "append", 32, 32, 128, "bf16", seqs=16, shortest=1, longest=1, lens_seed=0, page=16, bits=16, past=100, **_turn(False, 1, 128, start=190000)),
        # prompts quantised as they come, with norms
        _case("append_prompt_8bit", "append", 64, 8, 128, "bf16", seqs=4, shortest=2500, longest=4096, lens_seed=6, page=64, bits=8, past=0, **_turn(True, 1, 128, base=500000.0)),
        # the next pieces of prompts with images, three axes, half of each head turned; workload c3's width (1280 = 20 heads of 64)
        _case("append_images_f16", "append", 20, 20, 64, "f16", seqs=6, shortest=100, longest=1500, lens_seed=2, page=32, bits=16, past=600, **_turn(False, 3, 32, start=40)),
        # chunks of long documents that are read piece by piece
        _case("chunk_long_8bit", "chunk", 64, 8, 128, "bf16", seqs=4, shortest=400, longest=1024, lens_seed=3, page=256, bits=8, past=30000),
        # a mixed batch: chunks of prompts beside sequences that are sampled, in small pages
        _case("chunk_mixed_f16", "chunk", 32, 8, 128, "f16", seqs=12, shortest=1, longest=512, lens_seed=4, page=16, bits=16, past=4000),
        # a few drafted tokens of each of 24 sequences, looked over at once
        _case("chunk_drafts", "chunk", 32, 8, 128, "bf16", seqs=24, shortest=6, longest=6, lens_seed=5, page=64, bits=16, past=8192),
        # whole prompts of workload c4's width (4096 = 32 heads of 128), attended over as they were written
        _case("chunk_prompt", "chunk", 32, 32, 128, "bf16", seqs=2, shortest=4096, longest=4096, lens_seed=0, page=128, bits=16, past=0),
        # one short prompt after a few tokens: launch and latency
        _case("chunk_short", "chunk", 12, 12, 64, "bf16", seqs=1, shortest=17, longest=17, lens_seed=0, page=16, bits=16, past=200),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "append", "append", "chunk", "chunk", "chunk"])
    d = rng.choice([64, 128, 128, rng.choice([32, 80, 96, 112])])
    hkv = rng.choice([1, 2, 4, 8, 8, 12, 20, 32])
    hq = hkv * rng.choice([g for g in (1, 1, 2, 4, 8) if hkv * g <= 64])
    c = _case("", kind, hq, hkv, d, rng.choice(["bf16", "bf16", "f16"]), lens_seed=rng.randrange(1 << 30))
    c.pop("name")
    if kind != "chunk":
        c.update(_turn(rng.random() < 0.5, rng.choice([1, 1, 2, 3]), rng.choice([d, d, max(16, d // 32 * 16)]), rng.random() < 0.3, rng.choice([10000.0, 500000.0]),
                       rng.choice([0, 0, _log_uniform(rng, 1, 1 << 20)])))
    if kind == "rotary":
        longest = _log_uniform(rng, 1, 8192)
        most = min(16384 // longest, LARGEST_ROWS // ((hq + hkv) * d * longest))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, min(most, 32))), shortest=rng.choice([1, longest, max(1, longest // 4)]))
        return c
    c.update(page=rng.choice([16, 32, 64, 128, 256]), bits=rng.choice([16, 8]))
    if kind == "append":
        longest = rng.choice([1, _log_uniform(rng, 1, 4096)])
        past = rng.choice([0, _log_uniform(rng, 1, 600)])
        most = min(64, 16384 // (longest + past), LARGEST_ROWS // ((hq + hkv) * d * (longest + past)))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, most)), shortest=rng.choice([1, longest]), past=past)
    else:
        longest = rng.choice([_log_uniform(rng, 1, 16), _log_uniform(rng, 1, 4096), _log_uniform(rng, 1, 4096)])
        past = rng.choice([0, _log_uniform(rng, 1, 30000), _log_uniform(rng, 1, 30000)])
        most = min(64, 16384 // longest, LARGEST_CACHE // (hkv * d * (longest + past)), LARGEST_SCORES // (hq * d * longest * (longest + past)))
        c.update(longest=longest, seqs=_log_uniform(rng, 1, max(1, most)), shortest=rng.choice([1, longest, max(1, longest // 2)]), past=past)
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

    def normal(self, shape, dtype, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=self.gen, device="cuda") * std + mean).to(dtype)

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


def _positions(case, new, lens):
    """int32 [axes][new tokens]: text has the same position on all axes; of several axes, what follows the first 20 tokens is frames of 24 x 18 patches."""
    parts = []
    for n, k in zip(new, lens):
        at = torch.arange(k - n, k, device="cuda")
        if case["axes"] == 1:
            axes = [at]
        else:
            i = (at - 20).clamp(min=0)
            grid = [i // 432, i // 18 % 24, i % 18][3 - case["axes"]:]
            axes = [torch.where(at < 20, at, 20 + g) for g in grid]
        parts.append(torch.stack(axes))
    return (torch.cat(parts, 1) + case["start"]).to(torch.int32)


def _turning(case):
    """Frequency of each pair in 64 bits, and its axis: the axes have neighbouring pairs, the later ones as many as the first or one more."""
    pairs = case["rotated"] // 2
    i = torch.arange(pairs, dtype=torch.float64, device="cuda")
    return case["base"] ** (-i / pairs), (torch.arange(pairs, device="cuda") * case["axes"] // pairs).to(torch.int32)


def prepare(case, seed):
    rnd, dt, kind = _Inputs(seed), DTYPES[case["dtype"]], case["kind"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    new, lens = _lengths(case)
    n = sum(new)
    s = {"case": case, "new": new, "lens": lens, "cu": _on_gpu(_offsets(lens))}
    if kind != "chunk":   # views of one projection's result
        qkv = rnd.normal((n, hq + 2 * hkv, d), dt)
        qkv[:, hq:hq + hkv] = rnd.keys(n, hkv, d, dt)
        s["Q"], s["K"], s["V"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["w"] = [rnd.normal((d,), dt, 0.2, 1.0) if case["norm"] else None for _ in range(2)]
        s["positions"] = _positions(case, new, lens)
        s["frequencies"], s["axis"] = _turning(case)
    if kind == "rotary":
        dqkv = rnd.normal((n, hq + 2 * hkv, d), dt, 1e-2)
        s["dQ"], s["dK"] = dqkv[:, :hq], dqkv[:, hq:hq + hkv]
    else:
        s["pages"], s["table"], s["places"] = _paged(case, rnd, lens)
        K, V = rnd.keys(sum(lens), hkv, d, dt), rnd.normal((sum(lens), hkv, d), dt)
        if kind == "chunk":
            s["Q"] = rnd.normal((n, hq, d), dt)
            fill, written = slice(None), s["places"]
        else:   # the new ones are the last of each sequence
            is_new = torch.cat([torch.arange(k, device="cuda") >= k - m for k, m in zip(lens, new)])
            s["new_places"] = s["places"][is_new].contiguous()
            fill, written = ~is_new, s["places"][~is_new]
    if own:
        from paper_2404_01847_amd.attention import PagedKV, Rotary
        if kind != "chunk":
            s["rotary"] = Rotary(hq, hkv, d, n, s["frequencies"], *s["w"], eps=EPS, axis=s["axis"], axes=case["axes"], interleaved=case["interleaved"], dtype=dt)
        if kind != "rotary":
            s["cache"] = PagedKV(s["pages"], case["page"], hkv, d, dt, bits=case["bits"])
            s["cache"].write(K[fill].contiguous(), V[fill].contiguous(), written.contiguous())
        if kind == "chunk":
            s["cu_new"], s["lengths"], s["O"] = _on_gpu(_offsets(new)), _on_gpu(lens), torch.empty_like(s["Q"])
        if kind == "append":
            s["K_out"], s["V_out"] = torch.empty_like(K), torch.empty_like(V)
        if kind == "rotary":
            s["dQ_out"], s["dK_out"] = torch.empty_like(s["dQ"]), torch.empty_like(s["dK"])
    elif kind != "rotary":
        s["cache"] = [_plain_pages(s["pages"] * case["page"], hkv, d, dt, case["bits"]) for _ in range(2)]
        for held, x in zip(s["cache"], (K, V)):
            _plain_write(held, x[fill], written)
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_angles(s):
    """Cosine and sine [tokens][1][pairs] in 32 bits, of angles in 64."""
    at = s["positions"][s["axis"].long()].t().double() * s["frequencies"]
    return torch.cos(at).float()[:, None], torch.sin(at).float()[:, None]


def _plain_turn(x, cos, sin, case):
    """x [tokens][heads][d] in 32 bits, turned."""
    r = case["rotated"]
    out = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    return out


def _plain_normed(x, w):
    """Normalised x without its weights, and the factor of each row."""
    r = torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)
    return x * r, r


def _plain_forward(x, w, cos, sin, case):
    x = x.float()
    if w is not None:
        x = _plain_normed(x, w)[0] * w.float()
    return _plain_turn(x, cos, sin, case)


def _plain_backward(dz, x, w, cos, sin, case):
    g = _plain_turn(dz.float(), cos, -sin, case)
    if w is None:
        return g, None
    y, r = _plain_normed(x.float(), w)
    gw = g * w.float()
    return r * (gw - y * (gw * y).mean(2, keepdim=True)), (g * y).sum(1).sum(0)


def _plain_pages(places, hkv, d, dt, bits):
    if bits == 16:
        return {"values": torch.zeros((places, hkv, d), dtype=dt, device="cuda")}
    return {"values": torch.zeros((places, hkv, d), dtype=torch.int8, device="cuda"), "step": torch.zeros((places, hkv, 1), dtype=torch.float32, device="cuda")}


def _plain_write(held, x, places):
    if "step" not in held:
        held["values"][places] = x.to(held["values"].dtype)
        return
    x = x.float()
    s = (x.abs().amax(dim=2, keepdim=True) / 127).clamp(min=2.0 ** -126)
    held["values"][places] = torch.round(x / s).clamp(-127, 127).to(torch.int8)
    held["step"][places] = s


def _plain_read(held, places):
    x = held["values"][places].float()
    return x * held["step"][places] if "step" in held else x


def _plain_attention(q, k, v, group):
    """Of one sequence: q [lq][hq][d], k and v [lk][hkv][d] in 32 bits; a few heads at a time."""
    lq, hq, d = q.shape
    lk, hkv = k.shape[:2]
    O = torch.empty_like(q)
    hidden = torch.arange(lk, device=q.device)[None, :] > torch.arange(lq, device=q.device)[:, None] + (lk - lq)
    step = max(1, (1 << 28) // (lq * lk * group))
    for h in range(0, hkv, step):
        n = min(step, hkv - h)
        heads = slice(h * group, (h + n) * group)
        qh = q[:, heads].reshape(lq, n, group, d).permute(1, 2, 0, 3).reshape(n, group * lq, d)
        kh, vh = k[:, h:h + n].permute(1, 2, 0).contiguous(), v[:, h:h + n].permute(1, 0, 2).contiguous()
        P = torch.matmul(qh, kh).mul_(d ** -0.5).view(n, group, lq, lk)
        P.masked_fill_(hidden, -math.inf)
        P.sub_(P.amax(dim=3, keepdim=True)).exp_()
        P.div_(P.sum(dim=3, keepdim=True))
        O[:, heads] = torch.matmul(P.view(n, group * lq, lk), vh).view(n, group, lq, d).permute(2, 0, 1, 3).reshape(lq, n * group, d)
    return O


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if own:
        if kind == "rotary":
            Q, K = s["rotary"].forward(s["Q"], s["K"], s["positions"])
            dQ, dK = s["rotary"].backward(s["dQ"], s["dK"], s["Q"], s["K"], s["positions"], out=(s["dQ_out"], s["dK_out"]))
            return {"Q": Q, "K": K, "dQ": dQ, "dK": dK, **({"dwq": s["rotary"].dwq, "dwk": s["rotary"].dwk} if case["norm"] else {})}
        if kind == "chunk":
            return s["cache"].attend_chunk(s["Q"], s["cu_new"], s["table"], s["lengths"], s["O"])
        Q = s["cache"].append(s["rotary"], s["Q"], s["K"], s["V"], s["positions"], s["new_places"])
        s["cache"].read(s["table"], s["cu"], s["K_out"], s["V_out"])
        return {"Q": Q, "K": s["K_out"], "V": s["V_out"]}
    if kind == "chunk":
        q = s["Q"].float()
        O = torch.empty(q.shape, dtype=dt, device="cuda")
        a, b = _offsets(s["new"]), _offsets(s["lens"])
        for i in range(len(s["new"])):
            K, V = (_plain_read(held, s["places"][b[i]:b[i + 1]]) for held in s["cache"])
            O[a[i]:a[i + 1]] = _plain_attention(q[a[i]:a[i + 1]], K, V, case["hq"] // case["hkv"])
        return O
    cos, sin = _plain_angles(s)
    Q, K = (_plain_forward(x, w, cos, sin, case) for x, w in zip((s["Q"], s["K"]), s["w"]))
    if kind == "append":
        for held, x in zip(s["cache"], (K, s["V"])):
            _plain_write(held, x, s["new_places"])
        return {"Q": Q.to(dt), **{name: _plain_read(held, s["places"]).to(dt) for name, held in zip("KV", s["cache"])}}
    out = {"Q": Q.to(dt), "K": K.to(dt)}
    for name, dz, x, w in zip("QK", (s["dQ"], s["dK"]), (s["Q"], s["K"]), s["w"]):
        dx, dw = _plain_backward(dz, x, w, cos, sin, case)
        out["d" + name] = dx.to(dt)
        if dw is not None:
            out["dw" + name.lower()] = dw
    return out


# ---------------------------------------------------------------------------------------------------- what it takes
def _pairs(case):
    """Visible pairs of a query and a key, of one head."""
    new, lens = _lengths(case)
    return sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, lens))


def work(case):
    """Inputs read once and outputs written once; of the causal products the visible pairs."""
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    new, lens = _lengths(case)
    n = sum(new)
    if kind == "rotary":   # Q, K, dQ and dK in (without norms their gradients need no Q and K, which the forward pass has read); four out
        return {"bytes": n * (hq + hkv) * d * 2 * 4, "flops": n * (hq + hkv) * (3.0 * case["rotated"] * 2 + (15.0 * d if case["norm"] else 0.0))}
    held = 2 * hkv * (2 * d if case["bits"] == 16 else d + 4)   # bytes of a token in the cache
    if kind == "append":   # new tokens in, their queries out and their place in the cache; older ones from the cache; all keys and values of the sequences out
        return {"bytes": n * (2 * hq + 2 * hkv) * d * 2 + sum(lens) * (held + 2 * hkv * d * 2), "flops": 0}
    return {"bytes": sum(lens) * held + 2 * n * hq * d * 2, "flops": 4.0 * _pairs(case) * hq * d}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_heads(x, w, turn, case):
    """x [tokens][heads][d] in 64 bits: normalised, its pairs as complex numbers times e^(i angle)."""
    r = case["rotated"]
    if w is not None:
        x = x / (x.pow(2).sum(2, keepdim=True) / x.shape[2] + EPS).sqrt() * w.double()
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:2], r // 2, 2).contiguous()) * turn
        front = torch.view_as_real(z).reshape(*x.shape[:2], r)
    else:
        z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
        front = torch.cat([z.real, z.imag], 2)
    return torch.cat([front, x[..., r:]], 2)


def _exact_held(x, bits, dt):
    """What a cache holds of x [..., d], as the values it stands for."""
    if bits == 16:
        return x
    s = (x.abs().amax(dim=-1, keepdim=True) / 127).float().clamp(min=2.0 ** -126).double()
    return torch.round(x / s).clamp(-127, 127) * s


def exact(case, seed):
    global own
    if case["kind"] == "chunk" and case["seqs"] * case["hq"] > 4096:
        return None
    kept, own = own, False
    rnd, dt, kind = _Inputs(seed), DTYPES[case["dtype"]], case["kind"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    new, lens = _lengths(case)
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if kind != "chunk":
        angle = torch.stack([s["positions"][a].double() * f for a, f in zip(s["axis"].tolist(), s["frequencies"])], 1)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    if kind == "rotary":
        out = {}
        for name, x, dz, w in zip("QK", (s["Q"], s["K"]), (s["dQ"], s["dK"]), s["w"]):
            x = x.double().requires_grad_()
            w = None if w is None else w.double().requires_grad_()
            z = _exact_heads(x, w, turn, case)
            grads = torch.autograd.grad(z, [x] if w is None else [x, w], dz.double())
            out[name], out["d" + name] = z.detach(), grads[0]
            if w is not None:
                out["dw" + name.lower()] = grads[1]
        return out
    # the inputs of `prepare`, in its order
    if kind == "append":
        rnd.normal((sum(new), hq + 2 * hkv, d), dt), rnd.keys(sum(new), hkv, d, dt)
        if case["norm"]:
            rnd.normal((d,), dt), rnd.normal((d,), dt)
    _paged(case, rnd, lens)
    K, V = rnd.keys(sum(lens), hkv, d, dt).double(), rnd.normal((sum(lens), hkv, d), dt).double()
    if kind == "append":
        is_new = torch.cat([torch.arange(k, device="cuda") >= k - n for k, n in zip(lens, new)])
        K[is_new], V[is_new] = _exact_heads(s["K"].double(), s["w"][1], turn, case), s["V"].double()
        return {"Q": _exact_heads(s["Q"].double(), s["w"][0], turn, case), "K": _exact_held(K, case["bits"], dt), "V": _exact_held(V, case["bits"], dt)}
    K, V = _exact_held(K, case["bits"], dt), _exact_held(V, case["bits"], dt)
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    a, b = _offsets(new), _offsets(lens)
    for i in range(len(new)):
        for h in range(hq):
            k, v = K[b[i]:b[i + 1], h * hkv // hq], V[b[i]:b[i + 1], h * hkv // hq]
            t = torch.mm(s["Q"][a[i]:a[i + 1], h].double(), k.t()) / math.sqrt(d)
            seen = torch.arange(lens[i], device="cuda")[None] - torch.arange(new[i], device="cuda")[:, None] <= lens[i] - new[i]
            t = torch.where(seen, t, torch.full_like(t, -math.inf))
            O[a[i]:a[i + 1], h] = torch.mm(torch.exp(t - torch.logsumexp(t, dim=1, keepdim=True)), v)
    return O
