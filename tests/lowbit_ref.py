"""Plain 64-bit forms of the operators on the 8-bit cache and the microscaled 4-bit format, written from their definitions
(include/sun.h), and the tolerances that their tests share."""
from __future__ import annotations

import math

import numpy as np

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # half a step, relative to the value
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def _e4m3(code: int) -> float:
    e, m = code >> 3 & 15, code & 7
    v = math.nan if code & 127 == 127 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return -v if code & 128 else v


E4M3 = np.array([_e4m3(c) for c in range(256)])
_POS = E4M3[:127]


def to_e4m3(y):
    """Codes of numbers of magnitude up to 448, halves to the even code; 127 for what is not finite."""
    a = np.abs(np.where(np.isfinite(y), y, 0.0))
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    up = (a - _POS[lo] > _POS[hi] - a) | ((a - _POS[lo] == _POS[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, lo) | np.where(np.signbit(y), 128, 0)
    return np.where(np.isfinite(y), code, 127).astype(np.uint8)


def entry_exponent(top):
    """The smallest integer e >= -100 with top <= 448 * 2^e."""
    m, x = np.frexp(top)                      # top = m 2^x, 448 = 0.875 * 2^9
    return np.maximum(np.where(top > 0, x - 9 + (m > 0.875), -100), -100)


def entry(y):
    """Codes and scale bytes of vectors along the last axis."""
    e = entry_exponent(np.max(np.where(np.isfinite(y), np.abs(y), 0.0), -1))
    return to_e4m3(y * np.exp2(-e.astype(np.float64))[..., None]), (e + 127).astype(np.uint8)


def thetas(cfg):
    d = cfg.head_dim
    out = []
    for j in range(d // 2):
        t = float(cfg.rope_base) ** (-2.0 * j / d)
        if cfg.rope_scaling:
            turns = cfg.rope_original_max_position * t / (2 * math.pi)      # wavelengths in the original length
            low, high = cfg.rope_low_freq_factor, cfg.rope_high_freq_factor
            share = min(1.0, max(0.0, (turns - low) / (high - low)))
            t = t * share + t / cfg.rope_factor * (1 - share)
        out.append(t)
    return np.array(out)


def rotated(x, heads, cfg, positions, gain=None):
    """x [rows, heads * d] -> [rows, heads, d]: head norm, then rotation."""
    d = cfg.head_dim
    x = np.asarray(x, np.float64).reshape(-1, heads, d)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(cfg.rms_eps)) * np.asarray(gain, np.float64)
    ang = np.asarray(positions, np.float64)[:, None] * thetas(cfg)
    c, s = (f(ang).astype(np.float32).astype(np.float64)[:, None, :] for f in (np.cos, np.sin))
    a, b = x[..., :d // 2], x[..., d // 2:]
    with np.errstate(invalid="ignore"):
        return np.concatenate([a * c - b * s, b * c + a * s], -1)


def pool_views(mem, lay, n_layers, hkv, d):
    """Views of a host copy of the pool: k codes [layer, page, head, token, dim], v codes [layer, page, head, dim, token], scales of each
    [layer, page, head, token]."""
    def view(off, shape, strides):
        return np.lib.stride_tricks.as_strided(mem[off:], shape, strides)
    P = lay.n_pages
    return (view(lay.k_off, (n_layers, P, hkv, 16, d), (lay.k_layer, lay.k_page, lay.k_head, lay.k_token, lay.k_dim)),
            view(lay.v_off, (n_layers, P, hkv, d, 16), (lay.v_layer, lay.v_page, lay.v_head, lay.v_dim, lay.v_token)),
            view(lay.ks_off, (n_layers, P, hkv, 16), (lay.s_layer, lay.s_page, lay.s_head, 1)),
            view(lay.vs_off, (n_layers, P, hkv, 16), (lay.s_layer, lay.s_page, lay.s_head, 1)))


def attention(q, views, layer, table, n, window, hkv, n_pages):
    """One request: q [Hq, d] -> out [Hq, d] and, per element, sum_t p_t |v_t| and the score error scale max_t sum |q k_t| / sqrt d."""
    k_codes, v_codes, k_scales, v_scales = (v[layer] for v in views)
    hq, d = q.shape
    out, mass, reach = np.zeros((hq, d)), np.zeros((hq, d)), np.zeros(hq)
    seen = [t for t in range(max(0, n - window) if window else 0, n) if 0 <= table[t // 16] < n_pages]
    if not seen:
        return out, mass, reach
    page, slot = np.array([table[t // 16] for t in seen]), np.array(seen) % 16
    for h in range(hkv):
        k = E4M3[k_codes[page, h, slot]] * np.exp2(k_scales[page, h, slot].astype(np.float64) - 127)[:, None]
        v = E4M3[v_codes[page, h, :, slot]] * np.exp2(v_scales[page, h, slot].astype(np.float64) - 127)[:, None]
        for g in range(hq // hkv):
            i = h * (hq // hkv) + g
            s = k @ q[i] / math.sqrt(d)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i], mass[i] = p @ v, p @ np.abs(v)
            reach[i] = (np.abs(k) @ np.abs(q[i])).max() / math.sqrt(d)
    return out, mass, reach


def attention_bound(out, mass, reach, n, d, dtype):
    """Scores: d products summed in 32 bits and four roundings behind them; weights e^s off by twice that, an exponential good to 2^-22,
    carried in 16 (bf16) or 24 bits; two sums over n weights in 32 bits; the output's own rounding."""
    score = reach[..., None] * (d + 4) * 2.0 ** -24
    weight = 2 * score + 2.0 ** -21 + (2.0 ** -16 if dtype == "bf16" else 2.0 ** -24)
    return mass * (weight + 2 * (n + 8) * 2.0 ** -24) + np.abs(out) * HALF[dtype] * 1.01 + 1e-37


def mx4_quantize(x):
    x = np.asarray(x, np.float64)
    n, k = x.shape
    b = x.reshape(n, k // 32, 32)
    good = np.isfinite(b).all(-1)
    b = np.where(good[..., None], b, 0.0)
    top = np.abs(b).max(-1)
    e = np.maximum(np.where(top > 0, np.frexp(top)[1] - 3, -127), -127)
    y = b * np.exp2(-e.astype(np.float64))[..., None]
    a = np.minimum(np.abs(y), 6.0)
    hi = np.clip(np.searchsorted(E2M1[:8], a), 1, 7)
    up = (a - E2M1[hi - 1] > E2M1[hi] - a) | ((a - E2M1[hi - 1] == E2M1[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, hi - 1) | np.where(np.signbit(y), 8, 0)
    code = np.where(good[..., None], code, 0).reshape(n, k).astype(np.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, np.where(good, e + 127, 255).astype(np.uint8)


def mx4_values(codes, scales):
    n, half = codes.shape
    code = np.stack([codes & 15, codes >> 4], -1).reshape(n, -1, 32)
    power = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (E2M1[code] * power[..., None]).reshape(n, 2 * half)


def linear_bound(x, w, ref, dtype):
    """K products summed in 32 bits in any order, activations carried exactly, and the output's own rounding."""
    return (x.shape[1] + 8) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + np.abs(ref) * HALF[dtype] * 1.01 + 1e-37


# ------------------------------------------------------------------ what only the low bits of 32-bit attention decide

def close_queries(batch, heads, seed=8):
    """Pairs of 24-bit numbers in [2^20, 2^21) that differ in their last 8 bits alone; the 8 bits before those begin with a one, so that a cut behind
    the upper 8 and the next 8 bits leaves nothing of the difference."""
    rng = np.random.default_rng(seed)
    upper = (rng.integers(128, 256, (batch, heads)) << 8 | rng.integers(128, 256, (batch, heads))) << 8
    a, b = (rng.integers(0, 256, (batch, heads)) for _ in range(2))
    b = np.where(a == b, 255 - a, b)
    return tuple(((upper | x) / 8.0).astype(np.float32) for x in (a, b))


def cut(x, planes):
    """x as its first `planes` truncations to 8 significant bits add up to it."""
    left, total = np.asarray(x, np.float32), 0.0
    for _ in range(planes):
        top = (left.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        total, left = total + top.astype(np.float64), left - top
    return total


def close_queries_out(q_a, q_b, d):
    """Two tokens with scores (q_a - q_b) / sqrt d and 0 and values 1 and 0: the first one's weight, and how far 32 bits may be from it.  The products' partial
    sums are multiples of 2^-3 below 2^21 in any order, so q_a - q_b is exact.  The factor log2(e) / sqrt(d) is good to 2^-23, the product with the maximum and the
    fused one to 2^-24 each: s * 2^-22 of a weight; two exponentials to 2^-23, the weights' planes and sums to 2^-24 each, the quotient 2^-24: 2^-21 is more."""
    s = (np.asarray(q_a, np.float64) - np.asarray(q_b, np.float64)) / math.sqrt(d)
    out = 1 / (1 + np.exp(-s))
    return out, out * (np.abs(s) * 2.0 ** -22 + 2.0 ** -21)


def close_gaps(batch, heads, d, seed=9):
    """Queries whose scores against a key of one -1 are gaps of e^-0.5 to e^-0.01 between two weights."""
    return (np.random.default_rng(seed).uniform(0.01, 0.5, (batch, heads)) * math.sqrt(d)).astype(np.float32)


def close_gaps_out(q, d):
    """Two tokens with scores 0 and -g = -q / sqrt d, values 1 and -1: (1 - w) / (1 + w), w = e^-g in [0.6, 1), and how far 32 bits may be from it.  The first
    weight is 1.  The second is off by g * 2^-22 (see above), 2^-23 of its exponential and 2^-24 for its planes, the numerator by another 2^-24 and
    the denominator by 2^-24 of itself; the quotient rounds once more."""
    g = np.asarray(q, np.float64) / math.sqrt(d)
    w = np.exp(-g)
    out = (1 - w) / (1 + w)
    weight = w * (g * 2.0 ** -22 + 2.0 ** -23 + 2.0 ** -24)
    return out, ((1 + out) * weight + 2.0 ** -24) / (1 + w) + out * 2.0 ** -23
