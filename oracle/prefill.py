"""Oracle of a prefill's attention in float64 (test infrastructure only, see the package docstring).

An item has `past` tokens and n new ones behind them.  The query of new token i, at position p = past + i,
sees tokens j < min(past + n, max(p + 1, n_full)):

    s_j = scale * <q, k_j>,  o = sum_j softmax_j(s) v_j,  lse = log sum_j exp(s_j)

`attend` also returns what a bound on the rounding errors needs: sum_j softmax_j |v_j| for every output, and the
largest sum_d |q_d k_jd| of a row.
"""
import numpy as np


def sees(past, n, full):
    """How many tokens each new query sees."""
    p = past + np.arange(n)
    return np.minimum(past + n, np.maximum(p + 1, full))


def attend(q, k, v, past, full, scale):
    """q [n, heads, d], k and v [past + n, d], float64 -> o, lse, spread [n, heads, d], reach [n, heads]."""
    n, heads, _ = q.shape
    seen = sees(past, n, full)
    o, spread = np.zeros_like(q), np.zeros_like(q)
    lse, reach = np.zeros((n, heads)), np.zeros((n, heads))
    for i in range(n):
        kk, vv = k[:seen[i]], v[:seen[i]]
        s = scale * (q[i] @ kk.T)
        top = s.max(axis=1, keepdims=True)
        w = np.exp(s - top)
        total = w.sum(axis=1, keepdims=True)
        o[i], spread[i] = w @ vv / total, w @ np.abs(vv) / total
        lse[i] = (top + np.log(total))[:, 0]
        reach[i] = (np.abs(q[i]) @ np.abs(kk).T).max(axis=1)
    return o, lse, spread, reach


def turned(x, positions, axis_of_pair, freqs, layout, amplitude=1.0):
    """x [n, heads, d] float64; positions [n_axes, n]; pair i turned by positions[axis_of_pair[i]] * freqs[i]."""
    half = len(freqs)
    y = np.array(x, dtype=np.float64)
    for i in range(half):
        a, b = (i, i + half) if layout == "halves" else (2 * i, 2 * i + 1)
        angle = np.asarray(positions[axis_of_pair[i]], dtype=np.float64)[:, None] * float(freqs[i])
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
