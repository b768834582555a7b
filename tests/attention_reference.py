"""Attention in 64 bits on the CPU, and how far a result may be from it that rounds where the library says it does.

u = half a unit in the last place of the storage type, relative.  Rounded are: P and dS as operands (u each), the results (u), and O on its way into
delta.  The scores carry the error of an fp32 sum of d products, at most d 2^-24 sum|q||k|, which is a relative error of P; exp2, the sums of
P and the statistics add a few 2^-23.  With A_i = sum_j P_ij |v_j| and e the relative error of P, elementwise:
  |O - exact|  <= u |O| + (u + 2 e) A
  |dV - exact| <= u |dV| + (u + e') sum_i P_ij |dO_i|                                        (e': e, and that of lse)
  |dS - exact| <= E_ij = P_ij (sum|dO_i| (u |O_i| + (u + 2 e) A_i) + fp32) + (u + e') |dS_ij|
  |dQ - exact| <= u |dQ| + c E |K|,   |dK - exact| <= u |dK| + c E^T |Q|"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}   # half a step among the subnormals
OPERAND_TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}   # of P, dS and of weights as operands


def visible(lq, lk, causal):
    i, j = torch.arange(lq)[:, None], torch.arange(lk)[None, :]
    return (j <= i + lk - lq) if causal else torch.ones((lq, lk), dtype=torch.bool)


def head(q, k, v, scale, causal, dtype, dO=None):
    """One head of one sequence, float64 on the CPU: (O, lse, dQ, dK, dV) and the bounds of O, dQ, dK, dV (dK's and dV's without their own rounding:
    they are summed over heads)."""
    u, tiny = U[dtype], OPERAND_TINY[dtype]
    d, lq, lk = q.shape[1], q.shape[0], k.shape[0]
    seen = visible(lq, lk, causal)
    s = (q @ k.T * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1) if lk else torch.full((lq,), -math.inf, dtype=torch.float64)
    P = torch.exp(s - lse[:, None]).masked_fill(~seen, 0.0)
    O = P @ v
    size = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0)
    e = (d * 2.0 ** -24 * size.amax(1) if lk else torch.zeros(lq, dtype=torch.float64)) + 2.0 ** -20
    A = P @ v.abs()
    few = tiny * 256 * seen.sum(1)[:, None] * (v.abs().amax(0) if lk else 0.0)   # weights among the subnormals of binary16
    bO = (u + 2 * e[:, None]) * A + few
    out = {"O": O, "lse": lse, "bO": u * O.abs() + bO + TINY[dtype], "blse": 2 * e + 2.0 ** -22 * lse.abs()}
    if dO is not None:
        e2 = 3 * e[:, None] + 2.0 ** -22 * lse.abs().masked_fill(lse.isinf(), 0.0)[:, None]
        dP = dO @ v.T
        delta = (dO * O).sum(1, keepdim=True)
        dS = P * (dP - delta)
        fp32 = 2 * d * 2.0 ** -24 * (dO.abs() @ v.abs().T + (dO.abs() * O.abs()).sum(1, keepdim=True))
        E = P * ((dO.abs() * (u * O.abs() + bO)).sum(1, keepdim=True) + fp32) + (u + e2) * dS.abs() + tiny * seen
        out |= {"dQ": dS @ k * scale, "dK": dS.T @ q * scale, "dV": P.T @ dO}
        out |= {"bdQ": u * out["dQ"].abs() + scale * (E @ k.abs()) + TINY[dtype], "bdK": scale * (E.T @ q.abs()),
                "bdV": ((u + e2) * P + tiny * seen).T @ dO.abs()}
    return out


def packed(Q, K, V, cu_q, cu_k, scale, causal, dO=None):
    """All heads of packed sequences; dictionaries of results and bounds, laid out as the operands."""
    dtype, (tq, hq, d), hkv = Q.dtype, Q.shape, K.shape[1]
    f = lambda x: x.detach().cpu().double()
    Q, K, V, dO = f(Q), f(K), f(V), None if dO is None else f(dO)
    zero = lambda x: torch.zeros_like(x)
    r = {"O": zero(Q), "lse": torch.zeros((hq, tq), dtype=torch.float64)}
    b = {"O": zero(Q), "lse": torch.zeros((hq, tq), dtype=torch.float64)}
    if dO is not None:
        r |= {"dQ": zero(Q), "dK": zero(K), "dV": zero(V)}
        b |= {"dQ": zero(Q), "dK": zero(K), "dV": zero(V)}
    for i in range(len(cu_q) - 1):
        qs, ks = slice(cu_q[i], cu_q[i + 1]), slice(cu_k[i], cu_k[i + 1])
        for h in range(hq):
            g = h // (hq // hkv)
            x = head(Q[qs, h], K[ks, g], V[ks, g], scale, causal, dtype, None if dO is None else dO[qs, h])
            r["O"][qs, h], b["O"][qs, h], r["lse"][h, qs], b["lse"][h, qs] = x["O"], x["bO"], x["lse"], x["blse"]
            if dO is not None:
                r["dQ"][qs, h], b["dQ"][qs, h] = x["dQ"], x["bdQ"]
                for n in ("dK", "dV"):
                    r[n][ks, g] += x[n]
                    b[n][ks, g] += x["b" + n]
    for n in ("dK", "dV") if dO is not None else ():
        b[n] += U[dtype] * r[n].abs() + TINY[dtype]
    return r, b


def assert_within(got, ref, bound, what):
    got = got.detach().cpu().double()
    same = (got == ref) | ((got - ref).abs() <= bound)      # (infinities of lse are equal)
    if not bool(same.all()):
        at = tuple(int(x) for x in torch.nonzero(~same)[0])
        raise AssertionError(f"{what}: {int((~same).sum())} of {same.numel()} values off, first at {at}: {got[at].item()} for {ref[at].item()} +- {bound[at].item()}")


def quantise(x):
    """(whole numbers, steps) that the 8-bit cache holds of x [..., d], in 64 bits"""
    x = x.detach().cpu().double()
    s = (x.abs().amax(-1, keepdim=True) / 127).float().clamp(min=2.0 ** -126).double()
    return torch.round(x / s), s
