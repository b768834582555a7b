"""Norms and rotations of heads in 64 bits on the CPU, and how far a result may be from them that is computed in 32 bits and rounded once.

u = half a unit in the last place of the storage type, relative; f = 2^-24.  The sum of squares runs over 16 values in a lane and over up to 8 lanes (20 f, all terms positive), its mean, eps
and the inverse root add 4 f: the factor r is off by 14 f, y = x r w by 17 f < 2^-19.9.  An angle is off by 2^-22 (the fraction of a turn in 32 bits, its conversion and product), its
series by 2^-24 and their evaluation by 2^-23: cosine and sine by 2^-21.  A turned value z = y_a cos - y_b sin is off by less than 2^-19 (|y_a| + |y_b|) before it is rounded:
  |z - exact|  <= u |z| + 2^-19 (|y_a| + |y_b|)
Backward: g is dz turned back, off by e_g = 2^-20 (|dz_a| + |dz_b|);  with y = x r, G = g w and M = mean(G y) the latter off by e_M <= mean(e_g |w y| + 2^-18 |G y|):
  |dx - exact| <= u |dx| + r (|w| e_g + 2^-20 |G| + |y| (e_M + 2^-18 |M|)) + 2^-19 r (|G| + |y M|)
  |dw - exact| <= sum(e_g |y| + 2^-18 |g y|) + (rows + 300) f sum |g y|          (a sum of so many terms in any order)"""
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}   # half a step among the subnormals


def angles(positions, frequencies, axis):
    """[tokens][1][pairs], from positions [axes][tokens]"""
    at = positions.cpu().double()
    axes = at.shape[0]
    which = torch.zeros(len(frequencies), dtype=torch.long) if axis is None else torch.where((axis < 0) | (axis >= axes), axes - 1, axis).cpu().long()
    return (at[which].T * frequencies.cpu().double())[:, None]


def partner(x, rotated, interleaved):
    """Of each value the other one of its pair (zeros past the turned ones)."""
    out = torch.zeros_like(x)
    if interleaved:
        out[..., 0:rotated:2], out[..., 1:rotated:2] = x[..., 1:rotated:2], x[..., 0:rotated:2]
    else:
        h = rotated // 2
        out[..., :h], out[..., h:rotated] = x[..., h:rotated], x[..., :h]
    return out


def spread(v, rotated, d, interleaved, fill):
    """[tokens][1][pairs] -> of each value its pair's"""
    out = torch.full((*v.shape[:2], d), fill, dtype=torch.float64)
    if interleaved:
        out[..., 0:rotated:2], out[..., 1:rotated:2] = v, v
    else:
        out[..., :rotated // 2], out[..., rotated // 2:rotated] = v, v
    return out


def turned(y, angle, rotated, interleaved):
    d = y.shape[-1]
    c, s = spread(torch.cos(angle), rotated, d, interleaved, 1.0), spread(torch.sin(angle), rotated, d, interleaved, 0.0)
    sign = torch.ones(d, dtype=torch.float64)
    sign[slice(0, rotated, 2) if interleaved else slice(0, rotated // 2)] = -1.0
    return y * c + sign * partner(y, rotated, interleaved) * s


def forward(x, w, eps, angle, rotated, interleaved):
    """z, and its bound without the rounding to the storage type"""
    x = x.detach().cpu().double()
    y = x if w is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.detach().cpu().double()
    return turned(y, angle, rotated, interleaved), 2.0 ** -19 * (y.abs() + partner(y.abs(), rotated, interleaved))


def backward(dz, x, w, eps, angle, rotated, interleaved):
    """dx, dw, and their bounds, dx's without the rounding to the storage type"""
    dz = dz.detach().cpu().double()
    g, eg = turned(dz, -angle, rotated, interleaved), 2.0 ** -20 * (dz.abs() + partner(dz.abs(), rotated, interleaved))
    if w is None:
        return g, None, eg, None
    x, w = x.detach().cpu().double(), w.detach().cpu().double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    y, G = x * r, g * w
    M = (G * y).mean(-1, keepdim=True)
    eM = (eg * (w * y).abs() + 2.0 ** -18 * (G * y).abs()).mean(-1, keepdim=True)
    bound = r * (w.abs() * eg + 2.0 ** -20 * G.abs() + y.abs() * (eM + 2.0 ** -18 * M.abs())) + 2.0 ** -19 * r * (G.abs() + (y * M).abs())
    rows, size = x.shape[0] * x.shape[1], (g * y).abs().sum((0, 1))
    return r * (G - y * M), (g * y).sum((0, 1)), bound, (eg * y.abs()).sum((0, 1)) + 2.0 ** -18 * size + (rows + 300) * 2.0 ** -24 * size


def rounded(ref, bound, dtype):
    return bound + U[dtype] * (ref.abs() + bound) + TINY[dtype]
