"""fp64 oracle of what lies between a layer's projections and its attention: heads normalised and rotated, the gradients of that,
rows as a cache of 4-bit (or 8-bit) codes holds them.  Plain numpy from the definitions; shares no code with the library."""
import math

import numpy as np


def frequencies(rotary_dim, theta=1.0e6, scaling="plain", factor=1.0, original_positions=0, beta_fast=32.0, beta_slow=1.0):
    """(angle per position of every rotated pair, default attention factor)."""
    r, out = rotary_dim, []
    for i in range(r // 2):
        f = theta ** (-2.0 * i / r)
        if scaling == "linear":
            f = f / factor
        elif scaling == "ntk":
            f = (theta * factor ** (r / (r - 2.0))) ** (-2.0 * i / r)
        elif scaling == "yarn":
            edges = [r * math.log(original_positions / (n * 2.0 * math.pi)) / (2.0 * math.log(theta)) for n in (beta_fast, beta_slow)]
            lo, hi = max(math.floor(edges[0]), 0), min(math.ceil(edges[1]), r - 1)
            g = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = f * (1.0 - g) + f / factor * g
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1.0 if scaling == "yarn" and factor > 1.0 else 1.0)


def _pairs(rotary_dim, layout):
    i = np.arange(rotary_dim // 2)
    return (i, i + rotary_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(x, positions, freq, a, layout, back=False):
    """x[n, heads, D] with the pairs of its leading 2 len(freq) dims turned by positions[n] * freq, times a; back: the transposed map."""
    lo, hi = _pairs(2 * len(freq), layout)
    angle = positions[:, None, None].astype(np.float64) * freq
    c, s = a * np.cos(angle), (-a if back else a) * np.sin(angle)
    y = x.copy()
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y


def normalise(x, w, eps):
    if w is None:
        return x.copy()
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def norm_rope(x, w, positions, eps, freq, a, layout):
    return rotate(normalise(x, w, eps), positions, freq, a, layout)


def norm_rope_bwd(g, x, w, positions, eps, freq, a, layout):
    """(dx, dw) for the gradient g of norm_rope's result."""
    h = rotate(g, positions, freq, a, layout, back=True)
    if w is None:
        return h, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dx = r * h * w - x * r ** 3 * (h * w * x).mean(-1, keepdims=True)
    return dx, (h * x * r).sum((0, 1))


# ------------------------------------------------------------------ codes
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """fp64 values rounded once to bf16 (normal range), ties to even."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def block_exponent(amax, largest):
    """The smallest k from -100 on with amax <= largest * 2^k; 0 for amax = 0."""
    amax = np.asarray(amax, np.float64)
    k = np.full(amax.shape, -100)
    while True:
        short = amax > largest * np.ldexp(1.0, k)
        if not short.any():
            return np.where(amax == 0.0, 0, k)
        k = k + short


def mxfp4(x):
    """What the 4-bit cache holds for rows x[..., D]: the E2M1 values times 2^k of every block of 32 (ties to the even code); a block with an
    infinite or undefined element reads as NaN."""
    y = np.asarray(x, np.float64).reshape(-1, 32)
    bad = ~np.isfinite(y).all(1)
    y = np.where(bad[:, None], 0.0, y)
    k = block_exponent(np.abs(y).max(1), 6.0)[:, None]
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    gap = np.abs(np.ldexp(np.abs(y), -k)[..., None] - E2M1[even_first])
    out = np.copysign(np.ldexp(E2M1[even_first[gap.argmin(-1)]], k), y)
    out[bad] = np.nan
    return out.reshape(np.shape(x))
