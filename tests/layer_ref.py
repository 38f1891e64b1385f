"""Plain statements of the 8-bit linear layer with its epilogue and of the gated feed-forward block for the tests: what is
compared byte by byte step by step in float32, the rest in float64 with the bounds of what the kernels' roundings add up to.
Nothing of the library.

Bounds.  E = 2^-24 is half a unit of float32, relative.  The scale of a normed row: the sum of squares goes through at most
d/2048 + 18 roundings of positive terms, of which the square root takes half, and mean, eps, root, quotient and product add one
each: (d/2048 + 24) E is more than that.  A linear layer's value before its rounding to 16 bits: the conversion of the sum, two
scalings and a bias, 4 E of |sum| s u + |b|, and the scale's error.  Activations: at most 1.13 times their argument's error
(the largest slope of the four) and their own, as the header states it."""
import numpy as np
import torch
from scipy import special

import serving_ref as ref

F32 = np.float32
E = 2.0 ** -24
SLOPE = 1.13


def norm_quantize(x, g, eps):
    """x float32 [n][d], g float32 [d] or None -> int8 codes and float64 scales, both exact, and the scales' relative bound."""
    if g is None:
        codes, scale = ref.quantize_tokens(x)
        return codes, scale.astype(np.float64), 0.0
    with np.errstate(over="ignore"):
        v = (x * g).astype(F32)
    codes, s = ref.quantize_tokens(v)
    x64 = x.astype(np.float64)
    r = 1.0 / np.sqrt((x64 * x64).mean(1) + float(F32(eps)))
    return codes, s.astype(np.float64) * r, (x.shape[1] / 2048 + 24) * E


def act(z, name):
    """float64 value and the relative bound of the kernels' activation."""
    if name in (None, "none"):
        return z, 0.0
    if name == "relu":
        return np.maximum(z, 0), 0.0
    if name == "silu":
        return z * special.expit(z), (5 + np.abs(z)) * 2.0 ** -22
    if name == "gelu":
        return 0.5 * z * special.erfc(-z / np.sqrt(2)), (5 + z * z) * 2.0 ** -22
    w = np.sqrt(8 / np.pi) * (z + 0.044715 * z ** 3)
    return z * special.expit(w), (5 + 3 * np.abs(w)) * 2.0 ** -22


def linear(codes, scale, rel, w_codes, w_scale, bias):
    """float64 value of the layer before its activation, and its bound.  Sums of int8 products below 2^53 are exact in float64."""
    acc = codes.astype(np.float64) @ w_codes.astype(np.float64).T
    z = acc * scale[:, None] * w_scale[None].astype(np.float64)
    mag = np.abs(z)
    err = (4 * E + rel) * mag
    if bias is not None:
        b = bias.astype(np.float64)
        z, err = z + b, err + 4 * E * np.abs(b)
    return z, err


def activated(z, err, name):
    a, own = act(z, name)
    slope = 1.0 if name in (None, "none", "relu") else SLOPE
    return a, slope * err + own * np.abs(a) + 2.0 ** -100


def finish(z, err, name, residual, dtype):
    """The 16-bit output: value and bound."""
    y, err = activated(z, err, name)
    if residual is not None:
        r = residual.astype(np.float64)
        err = err + E * (np.abs(y) + np.abs(r))
        y = y + r
    return y, err + ref.half_ulp(np.abs(y) * (1 + 2.0 ** -7) + err, dtype)


def _round16(v, dtype):
    return torch.from_numpy(v).to(dtype).float().numpy()


def gated(x, g, eps, gate, up, down, name, residual, dtype):
    """gate, up, down: (codes, scale, bias) in numpy.  The value of y and its bound: h lies between the 16-bit neighbours of its
    value's bounds, nearly always one and the same, and where it does not, its code and the row's scale lie between theirs."""
    codes, scale, rel = norm_quantize(x, g, eps)
    zg, eg = linear(codes, scale, rel, *gate)
    zu, eu = linear(codes, scale, rel, *up)
    a, ea = activated(zg, eg, name)
    p = a * zu
    ep = ea * np.abs(zu) + np.abs(a) * eu + ea * eu + 3 * E * np.abs(p) + 2.0 ** -100
    mid, lo, hi = _round16(p, dtype), _round16(p - ep, dtype), _round16(p + ep, dtype)
    least = np.where(lo * hi <= 0, 0, np.minimum(np.abs(lo), np.abs(hi))).max(1)
    most = np.maximum(np.abs(lo), np.abs(hi)).max(1)

    def values(h, amax):
        s = (amax.astype(F32) * ref.K127).astype(F32)
        s[amax < 2.0 ** -120] = 0
        inv = np.zeros_like(s)
        np.divide(F32(1), s, out=inv, where=s > 0)
        c = np.clip(np.rint((h * inv[:, None]).astype(F32)), -127, 127)
        return c.astype(np.float64), s[:, None].astype(np.float64)

    codes, scale = values(mid, np.abs(mid).max(1))
    held = codes * scale
    ends = np.stack([np.multiply(*values(h, m)) for h in (lo, hi) for m in (least, most)] + [held])
    spread = np.maximum(ends.max(0) - held, held - ends.min(0))
    wc, ws, bias = down
    # the sum of integers is exact in float64, which a sum of scaled codes would not be: it may be 0
    y = codes @ wc.astype(np.float64).T * scale * ws
    err = 4 * E * np.abs(y) + spread @ np.abs(wc).astype(np.float64).T * ws
    if bias is not None:
        b = bias.astype(np.float64)
        y, err = y + b, err + 4 * E * np.abs(b)
    return finish(y, err, None, residual, dtype)
