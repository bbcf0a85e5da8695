"""Norms of queries and keys with rotary positions, from their definition, in 64 bits, in plain numpy on the host."""
import numpy as np

import serving_plain as sp


def forward(x, w, positions, frequency, interleaved, amplitude, eps):
    """x [tokens, heads, dim]; frequency None: not turned.  Returns y and x r w."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return (y if frequency is None else sp.rotate(y, positions, frequency, interleaved, amplitude)), y


def pair_sums(x, frequency, interleaved, amplitude):
    """Where a result of the rotation has two terms, the sum of their magnitudes (with the cosine and the sine as 1)."""
    a = np.abs(x)
    if frequency is None:
        return a
    half = len(frequency)
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out = a.copy()
    out[..., i] = out[..., j] = (a[..., i] + a[..., j]) * abs(amplitude)
    return out


def gradients(x, w, g, positions, frequency, interleaved, amplitude, eps):
    """(dx, dw) of <y, g>, and the magnitudes of what they are summed from."""
    turned = g if frequency is None else sp.rotate(g, positions, frequency, interleaved, amplitude, inverse=True)
    big = pair_sums(g, frequency, interleaved, amplitude)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    unit = x * r
    dx = r * (w * turned - unit * (w * turned * unit).mean(-1, keepdims=True))
    size = r * (np.abs(w) * big + np.abs(unit) * (np.abs(w) * big * np.abs(unit)).mean(-1, keepdims=True))
    return dx, (turned * unit).sum((0, 1)), size, (big * np.abs(unit)).sum((0, 1))
