"""Float64 reference of the query/key head operators (test infrastructure only; shares no code with the library).

  frequencies    theta^(-2i/r) and its rescalings for contexts longer than the trained one
  rotate         position rotation of the first r elements of head rows, half or interleaved pairs
  norm_rotate    per-row RMS norm with a weight, rotation, R_3 (Sylvester-Hadamard / sqrt(d), Appendix A)
  norm_rotate_grad   the gradients of the heads and of the weight, from the formulas
"""
import math

import numpy as np

from . import conqur_oracle as O


def frequencies(r, theta=10000.0, scaling="none", factor=1.0, low=0.0, high=0.0, original=0):
    out = []
    for i in range(r // 2):
        base = theta * factor ** (r / (r - 2.0)) if scaling == "ntk" and r > 2 else theta
        f = base ** (-2.0 * i / r)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            turns = original * f / (2.0 * math.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                share = (turns - low) / (high - low)
                f = share * f + (1.0 - share) * f / factor
        elif scaling == "ramp":
            where = lambda t: r * math.log(original / (2.0 * math.pi * t)) / (2.0 * math.log(theta))  # noqa: E731
            a, b = max(math.floor(where(high)), 0), min(math.ceil(where(low)), r - 1)
            g = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = f * (1.0 - g) + f / factor * g
        out.append(f)
    return np.array(out), (1.0 + 0.1 * math.log(factor) if scaling == "ramp" else 1.0)


def rotate(x, pos, freq, amp, layout, sign=1.0):
    """x (n, heads, d) float64, pos (n,) integers."""
    x = np.array(x, dtype=np.float64)
    h = len(freq)
    if h == 0:
        return x
    # integers times a double lose bits at far positions: the product in extended precision, reduced there
    ang = pos.astype(np.longdouble)[:, None] * (freq.astype(np.longdouble) / (2.0 * np.pi))
    ang = 2.0 * np.pi * (ang - np.floor(ang)).astype(np.float64)
    c, s = amp * np.cos(ang)[:, None, :], sign * amp * np.sin(ang)[:, None, :]
    ia, ib = (np.arange(h), np.arange(h) + h) if layout == "half" else (2 * np.arange(h), 2 * np.arange(h) + 1)
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
    return x


def hadamard(x):
    shape = x.shape
    return O.hadamard_rows(x.reshape(-1, shape[-1])).reshape(shape)


def norm_rotate(x, w, eps, pos, freq, amp, layout, r3):
    """w None: no norm."""
    x = np.asarray(x, dtype=np.float64)
    if w is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * w
    y = rotate(x, pos, freq, amp, layout)
    return hadamard(y) if r3 else y


def rotate_inverse(y, pos, freq, amp, layout, r3):
    y = np.asarray(y, dtype=np.float64)
    return rotate(hadamard(y) if r3 else y, pos, freq, amp, layout, -1.0)


def norm_rotate_grad(dy, x, w, eps, pos, freq, amp, layout, r3):
    g = rotate_inverse(dy, pos, freq, amp, layout, r3)
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    dw = np.sum(g * x * r, axis=(0, 1))
    wg = w * g
    return r * (wg - x * r * r * np.mean(wg * x, axis=-1, keepdims=True)), dw
