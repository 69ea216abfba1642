"""GELU in the product's epilogue where its value is small: x times the normal distribution's lower tail, relative to itself."""
import math

import numpy as np
import pytest
import torch

from paper_2603_02599_amd import binding as sun
from test_gpu_mx4_epilogue import DEV, check, run_fused, run_gated

pytestmark = pytest.mark.gpu


def tail(x):
    """The normal distribution's upper tail at |x|, 64 bits."""
    return np.vectorize(lambda v: 0.5 * math.erfc(abs(v) / math.sqrt(2)), otypes=[float])(x)


def gelu(x):
    """The value, and how far 32 bits may be from it.  The tail is e^(-x^2/2) R(|x|).  The exponential's argument rounds three times (the square, the constant, their product), which takes 3 x^2/2 2^-24 of it,
    and the exponential itself 2^-22.  R is t P(t), t = 1 / (1 + a |x|), P of degree 7: 4e-7 off with its roundings, and t, off by 2^-23, makes 2.7 times that of it; three products
    2^-24 each: 4e-7 + 3.3e-7 + 1.8e-7 + 2.4e-7 < 2^-19.  Above 0 it is taken from x, which rounds once."""
    q = tail(x)
    out = np.where(x > 0, x - x * q, x * q)
    return out, np.abs(x) * q * (1.5 * x * x * 2.0 ** -24 + 2.0 ** -19) + np.abs(out) * 2.0 ** -24


@pytest.mark.parametrize("rows", [16, 128, 400])
def test_small_values_keep_their_digits(rows):
    k, n = 32, 24
    w = torch.zeros(n, k, device=DEV)
    w[:, 0] = 1
    w = sun.sun_mx4_quantize(w)
    y = np.concatenate([np.linspace(-13, 0, 900), -np.geomspace(1e-8, 13, 300), np.linspace(0, 6, 300)]).astype(np.float32)
    for at in range(0, len(y), rows):
        part = y[at:at + rows]
        x = torch.zeros(len(part), k, device=DEV)
        x[:, 0] = torch.from_numpy(part)
        ref, off = (np.repeat(v[:, None], n, 1) for v in gelu(part.astype(np.float64)))
        check(run_fused(w, x, torch.empty(len(part), n, device=DEV), activation=sun.SUN_ACT_GELU), ref, off, "f32")
        check(run_fused(w, x, torch.empty(len(part), n, device=DEV, dtype=torch.bfloat16), activation=sun.SUN_ACT_GELU), ref, off, "bf16")
        u = torch.zeros(n, k, device=DEV)
        u[:, 1] = 1
        x[:, 1] = 3.0   # exact, as the products are
        check(run_gated(w, sun.sun_mx4_quantize(u), x, torch.empty(len(part), n, device=DEV), activation=sun.SUN_ACT_GELU), 3 * ref, 3 * off + np.abs(ref) * 2.0 ** -22, "f32")
