"""Oracle of rotary positions in float64 (test infrastructure only, see the package docstring).

Pair i of a row's first r dims is a complex number that is multiplied by amplitude * exp(j position *
freqs[i]); pairs are (i, i + r/2) or (2i, 2i + 1), the other dims are copied.
"""
import math

import numpy as np


def turned(x, positions, freqs, layout, amplitude=1.0):
    """x [n, heads, d] float64, positions [n], layout "halves" or "pairs"."""
    half = len(freqs)
    r = 2 * half
    y = np.array(x, dtype=np.float64)
    a, b = (slice(0, half), slice(half, r)) if layout == "halves" else (slice(0, r, 2), slice(1, r, 2))
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(freqs, dtype=np.float64)
    z = (x[..., a] + 1j * x[..., b]) * (amplitude * np.exp(1j * angle))
    y[..., a], y[..., b] = z.real, z.imag
    return y


def frequencies(base, r, kind="plain", factor=1.0, low=0.0, high=0.0, original_len=0):
    """(frequencies, amplitude), pair by pair."""
    out = []
    for i in range(r // 2):
        b = base * factor ** (r / (r - 2)) if kind == "base" and r > 2 else base
        f = 1.0 / b ** (2 * i / r)
        turns = original_len * f / (2 * math.pi)
        if kind == "linear":
            f /= factor
        elif kind == "bands":
            if turns <= low:
                f /= factor
            elif turns < high:
                t = (turns - low) / (high - low)
                f = (1 - t) * f / factor + t * f
        elif kind == "ramp":
            pair = lambda n: r * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(0, math.floor(pair(high))), min(r - 1, math.ceil(pair(low)))
            t = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * (1 - t) + f / factor * t
        out.append(f)
    return np.array(out), 1.0 + 0.1 * math.log(factor) if kind == "ramp" else 1.0
