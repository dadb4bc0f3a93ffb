"""Oracle of the operators around the routed experts: plain numpy in 64 bits, no code of the GPU path.

``e4m3`` values are handled as numbers; ``e4m3_decode`` turns codes (uint8) into them.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
AMAX_FLOOR = np.float32(2.0 ** -100)


# ---- routing -------------------------------------------------------------------------------------

def route_scored(logits, bias, top_k, softmax=False, n_groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    """ids [T,k] int32, gate [T,k] float64, counts, offsets, perm; one token at a time, by sorting."""
    logits = np.asarray(logits, np.float32)
    t, e = logits.shape
    ids, gate = np.zeros((t, top_k), np.int32), np.zeros((t, top_k))
    size = e // n_groups
    for i in range(t):
        l = logits[i].astype(np.float64)
        nan = np.isnan(l)
        l[nan] = -np.inf
        with np.errstate(over="ignore", invalid="ignore"):
            if softmax:
                z = np.where(l == l.max(), 1.0, np.exp(l - l.max()))
                s = z / z.sum()
            else:
                s = 1.0 / (1.0 + np.exp(-l))
            value = s if bias is None else s + np.asarray(bias, np.float32).astype(np.float64)
        value = value.copy()
        if bias is not None:
            value[nan | np.isnan(value)] = -np.inf
        choice = l if bias is None else value
        allowed = np.ones(e, bool)
        if n_groups > 1 and top_groups < n_groups:
            worth = []
            for g in range(n_groups):
                part = slice(g * size, (g + 1) * size)
                if group_top == 1:
                    w = choice[part].max()
                else:
                    two = np.sort(value[part])[-2:]
                    with np.errstate(invalid="ignore"):
                        w = two[0] + two[1]
                worth.append(-np.inf if np.isnan(w) else w)
            keep = sorted(range(n_groups), key=lambda g: (-worth[g], g))[:top_groups]
            allowed[:] = False
            for g in keep:
                allowed[g * size:(g + 1) * size] = True
        order = sorted(np.flatnonzero(allowed), key=lambda x: (-choice[x], x))[:top_k]
        ids[i] = order
        w = s[order]
        gate[i] = scale * (w / (w.sum() + 1e-20) if renormalise else w)
    flat = ids.reshape(-1)
    counts = np.bincount(flat, minlength=e).astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    perm = np.argsort(flat, kind="stable").astype(np.int32)
    return ids, gate, counts, offsets, perm


# ---- e4m3 with a scale per 128 -------------------------------------------------------------------

def _e4m3_table():
    v = np.zeros(256)
    for c in range(256):
        sign, exp, man = (-1.0 if c & 0x80 else 1.0), (c >> 3) & 15, c & 7
        v[c] = sign * (man * 2.0 ** -9 if exp == 0 else (1 + man / 8) * 2.0 ** (exp - 7))
    v[0x7F] = v[0xFF] = np.nan
    return v


E4M3 = _e4m3_table()


def e4m3_decode(codes):
    return E4M3[np.asarray(codes, np.uint8)]


def e4m3_encode(v):
    """The nearest e4m3 code of numbers, ties to even, beyond 448 clamped; NaN: 0x7f."""
    v = np.asarray(v, np.float64)
    table = E4M3[:127]                                    # ascending magnitudes of codes 0 .. 126
    mag = np.minimum(np.abs(np.where(np.isnan(v), 0.0, v)), 448.0)
    hi = np.clip(np.searchsorted(table, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - mag, mag - table[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(np.signbit(v), code | 0x80, code).astype(np.uint8)
    return np.where(np.isnan(v), np.uint8(0x7F), code)


def block_amax(v):
    """Largest magnitudes per row and 128 columns, at least 2^-100; NaN where a block holds one."""
    v = np.asarray(v)
    cols = v.shape[1]
    pad = np.zeros((v.shape[0], -cols % BLOCK), v.dtype)
    b = np.abs(np.concatenate([v, pad], axis=1)).reshape(v.shape[0], -1, BLOCK)
    return np.maximum(b.max(axis=2), AMAX_FLOOR.astype(v.dtype))


def quantize(v):
    """fp32 values to (codes, scales): each step one fp32 operation, as the interface states them."""
    v = np.asarray(v, np.float32)
    amax = block_amax(v)
    with np.errstate(invalid="ignore", over="ignore"):
        inverse = np.float32(448.0) / amax
        scaled = v * np.repeat(inverse, BLOCK, axis=1)[:, :v.shape[1]]
        return e4m3_encode(scaled), amax / np.float32(448.0)


def dequantize(codes, scales):
    codes = np.asarray(codes)
    with np.errstate(invalid="ignore"):
        return e4m3_decode(codes) * np.repeat(np.asarray(scales, np.float64), BLOCK, axis=1)[:, :codes.shape[1]]


def swiglu(x):
    x = np.asarray(x, np.float64)
    gate, up = x[:, :x.shape[1] // 2], x[:, x.shape[1] // 2:]
    with np.errstate(over="ignore", invalid="ignore"):
        return gate / (1.0 + np.exp(-gate)) * up


# ---- norms ---------------------------------------------------------------------------------------

def rms(v, eps):
    with np.errstate(over="ignore", invalid="ignore"):
        return v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


def norm_residual(x, y, post, gate, pre, gate_tokens, eps, residual_scale):
    """(x', h, the addend residual_scale * gate * z) in float64; y, post, gate, pre may be None."""
    x = np.asarray(x, np.float64)
    step = np.zeros_like(x)
    if y is not None:
        z = np.asarray(y, np.float64)
        if post is not None:
            z = rms(z, eps) * np.asarray(post, np.float64)
        if gate is not None:
            rows = np.arange(x.shape[0]) // gate_tokens if gate_tokens > 0 else np.zeros(x.shape[0], int)
            z = z * np.asarray(gate, np.float64)[rows]
        step = float(np.float32(residual_scale)) * z
    out = x + step
    return out, None if pre is None else rms(out, eps) * np.asarray(pre, np.float64), step


# ---- products ------------------------------------------------------------------------------------

def matmul(a_codes, a_scale, b_codes, b_scale, add=None):
    """(result, sum of the terms' magnitudes) in float64."""
    a = dequantize(a_codes, a_scale)
    b = e4m3_decode(b_codes) * np.repeat(np.repeat(np.asarray(b_scale, np.float64), BLOCK, axis=0)[:b_codes.shape[0]],
                                         BLOCK, axis=1)[:, :b_codes.shape[1]]
    out, size = a @ b.T, np.abs(a) @ np.abs(b).T
    if add is not None:
        out, size = out + np.asarray(add, np.float64), size + np.abs(np.asarray(add, np.float64))
    return out, size
