"""Plain 64-bit (and, where bytes are compared, step-by-step 32-bit) statements of the 8-bit serving operators for
the tests: numpy on the CPU, nothing of the library."""
import numpy as np
import torch

F32 = np.float32
K127 = F32(1.0) / F32(127.0)
SCALE_LO, SCALE_HI = F32(2.0 ** -60), F32(2.0 ** 60)


def half_ulp(y, dtype):
    """Half a unit in the last place of the 16-bit dtype at |y|, as float64."""
    mant, tiny = (8, 2.0 ** -133) if dtype == torch.bfloat16 else (11, 2.0 ** -24)
    e = np.floor(np.log2(np.maximum(np.abs(y), 1e-300)))
    return np.maximum(0.5 * 2.0 ** (e + 1 - mant), 0.5 * tiny)


def quantize_tokens(x):
    """x float32 [n][d] -> int8 codes, float32 scales; every step one float32 operation."""
    amax = np.abs(x).max(1).astype(F32)
    scale = (amax * K127).astype(F32)
    scale[amax < F32(2.0 ** -120)] = 0
    inv = np.zeros_like(scale)
    np.divide(F32(1.0), scale, out=inv, where=scale > 0)
    return np.clip(np.rint((x * inv[:, None]).astype(F32)), -127, 127).astype(np.int8), scale


def linear(codes, scale, w_codes, w_scale, bias):
    """float64 product and the magnitude that its float32 roundings are relative to."""
    acc = codes.astype(np.int64) @ w_codes.astype(np.int64).T
    y = acc.astype(np.float64) * scale[:, None].astype(np.float64) * w_scale[None].astype(np.float64)
    mag = np.abs(y)
    if bias is not None:
        y, mag = y + bias.astype(np.float64), mag + np.abs(bias.astype(np.float64))
    return y, mag


def rotate(x, pos, cos, sin, interleaved):
    """x float32 [n][h][d]; the products, sums and differences of the rotation in float32, one rounding each."""
    rot, y = 2 * cos.shape[1], x.copy()
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s = cos[pos][:, None, :], sin[pos][:, None, :]
    y[..., a] = (x[..., a] * c).astype(F32) - (x[..., b] * s).astype(F32)
    y[..., b] = (x[..., b] * c).astype(F32) + (x[..., a] * s).astype(F32)
    return y


def append(cache, off, lens, table, k, v, cos=None, sin=None, interleaved=False):
    """cache: dict of k_codes, k_scale, v_codes, v_scale (numpy, changed in place); k, v float32 [n][h][d]."""
    P = cache["k_codes"].shape[2]
    for s, length in enumerate(lens):
        n = off[s + 1] - off[s]
        start = length - n
        for page in range(start // P, -(-length // P)) if n else ():
            lo, hi = max(start, page * P), min(length, (page + 1) * P)
            rows = slice(off[s] + lo - start, off[s] + hi - start)
            at, held = table[s][page], lo - page * P
            for name, x in (("k", k), ("v", v)):
                x = x[rows]
                if name == "k" and cos is not None:
                    x = rotate(x, np.arange(lo, hi), cos, sin, interleaved)
                codes, scale = cache[name + "_codes"][at], cache[name + "_scale"][at]
                for h in range(x.shape[1]):
                    before = scale[h] if held else F32(0)
                    step = F32(np.abs(x[:, h]).max() * K127)
                    after = max(before, min(max(step, SCALE_LO), SCALE_HI))
                    inv = F32(1) / after
                    if after > before and held:
                        codes[h, :held] = np.rint(codes[h, :held].astype(F32) * F32(before * inv))
                    codes[h, held: held + hi - lo] = np.clip(np.rint(x[:, h] * inv), -127, 127)
                    scale[h] = after


def attend(cache, off, lens, table, q, scale, causal=True, window=0):
    """float64 out [n][heads][d], lse [n][heads], and per output the two magnitudes that its errors are relative to:
    sum_j p_j |v_j| and max_j |v_j| times the number of visible keys; per row the bound of |score| terms
    scale * sum_e |q_e k_e|, maximum over the keys."""
    n, heads, d = q.shape
    H, P = cache["k_codes"].shape[1], cache["k_codes"].shape[2]
    g = heads // H
    out, lse = np.zeros((n, heads, d)), np.full((n, heads), -np.inf)
    weight, span, terms = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros((n, heads))
    for s, length in enumerate(lens):
        if length <= 0:
            continue
        ids = np.asarray(table[s][: -(-length // P)])
        kv = {x: (cache[x + "_codes"][ids].astype(np.float64) * cache[x + "_scale"][ids].astype(np.float64)[..., None, None])
              .transpose(0, 2, 1, 3).reshape(-1, H, d)[:length] for x in "kv"}
        for t in range(off[s], off[s + 1]):
            p = length - off[s + 1] + t
            hi = min(length, p + 1) if causal else length
            lo = max(0, p - window + 1) if window else 0
            if hi <= lo:
                continue
            for h in range(heads):
                k, v = kv["k"][lo:hi, h // g], kv["v"][lo:hi, h // g]
                x = q[t, h].astype(np.float64)
                sc = scale * (k @ x)
                w = np.exp(sc - sc.max())
                lse[t, h] = sc.max() + np.log(w.sum())
                w /= w.sum()
                out[t, h] = w @ v
                weight[t, h] = w @ np.abs(v)
                span[t, h] = np.abs(v).max() * (hi - lo)
                terms[t, h] = scale * (np.abs(k) @ np.abs(x)).max()
    return out, lse, weight, span, terms
