"""Plain float64 forms of the operators around the head (numpy, CPU), written from their definitions."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U24 = 2.0 ** -24          # half a unit in the last place of float32, relative


def padded(d: int) -> int:
    return -(-d // 128) * 128


def mx4_quantize(x: np.ndarray):
    """(codes, scales) of the rows of x (float64 holding the input's values), block by block and value by value."""
    R, d = x.shape
    dp = padded(d)
    v = np.zeros((R, dp))
    v[:, :d] = x
    v = v.reshape(R, dp // 32, 32)
    bad = ~np.isfinite(v).all(-1)
    amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(-1))
    _, ex = np.frexp(amax)                                  # amax = f 2^ex, f in [1/2, 1)
    e = np.where(amax == 0, -127, np.clip(ex - 1 - 2, -127, 127))
    with np.errstate(invalid="ignore"):
        q = np.abs(v) / (2.0 ** e.astype(np.float64))[..., None]
    dist = np.abs(np.minimum(np.where(np.isfinite(q), q, 0.0), 6.0)[..., None] - GRID)
    near = dist == dist.min(-1, keepdims=True)              # one value, or two where it lies half way
    first = near.argmax(-1)
    second = 7 - near[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, second) | (np.signbit(v).astype(np.int64) << 3)
    code = np.where(bad[..., None], 0, code).astype(np.uint8).reshape(R, dp // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def mx4_values(codes: np.ndarray, scales: np.ndarray, d: int) -> np.ndarray:
    R = codes.shape[0]
    code = np.stack([codes & 15, codes >> 4], -1).reshape(R, -1, 32)
    v = GRID[code & 7] * np.where(code >> 3, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(R, -1)[:, :d]


def rows_logp(x: np.ndarray, tokens: np.ndarray, c: float):
    """Per row: m, s, logp; and p [N, V].  x float64."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = x.max(1)
        e = np.where(np.isneginf(m)[:, None], np.where(np.isnan(x), np.nan, 0.0), np.exp(c * (x - m[:, None])))
        s = e.sum(1)
        xt = x[np.arange(len(x)), np.clip(tokens, 0, x.shape[1] - 1)]
        logp = np.where(s == 0, -np.inf, c * (xt - m) - np.log(s))
        return m, s, logp, np.where(s[:, None] == 0, 0.0, e / s[:, None])


def out_of_range(tokens, V):
    return (tokens < 0) | (tokens >= V)


def grad_rows(p: np.ndarray, s: np.ndarray, tokens: np.ndarray, g: np.ndarray, c: float) -> np.ndarray:
    """c g ([j = t] - p); zeros where the row is left out, has no distribution or g is 0."""
    N, V = p.shape
    out = -p.copy()
    ok = ~out_of_range(tokens, V)
    out[np.arange(N)[ok], tokens[ok]] += 1.0
    with np.errstate(invalid="ignore"):
        out *= c * g[:, None]
    out[~ok | (s == 0) | (g == 0)] = 0.0
    return out


def policy(logp, old, ref, adv, w, lo, hi, beta):
    """Per row: the weighted loss term and its derivative by logp."""
    with np.errstate(invalid="ignore", over="ignore"):
        r = np.exp(logp - old)
        t = -np.minimum(r * adv, np.clip(r, 1 - lo, 1 + hi) * adv)
        d = np.where(np.where(adv >= 0, r <= 1 + hi, r >= 1 - lo), -adv * r, 0.0)
        if beta > 0:
            k = ref - logp
            t = t + beta * (np.exp(k) - k - 1)
            d = d + beta * (1 - np.exp(k))
        return w * t, w * d


def logp_tolerance(x, m, p, c, logp):
    """How far a float32 evaluation of logp may be off, per row.

    A term exp(c (x - m)) carries: the difference, c log2(e) and the product rounded to float32 and log2(e) itself, 4 U24 of its
    argument; the exponential, one unit, 2 U24.  The sum in any order of at most 256 additions per thread and a tree of 10: 266 U24,
    the rescaling of a running sum as often again.  The result is rounded once."""
    a = np.abs(c * (np.where(np.isfinite(x), x, m[:, None]) - m[:, None]))
    rel = (p * (4 * a + 2)).sum(1) * U24 + 532 * U24
    return rel + np.abs(logp) * U24, rel


def bf16_values(t):
    """float64 numpy values of a CPU tensor."""
    return t.double().numpy()
