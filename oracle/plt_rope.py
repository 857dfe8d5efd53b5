"""fp64 CPU oracle of the norm and rotation of queries and keys (test infrastructure only; the product never imports it): one
head's row at a time, a pair as a complex number."""
from __future__ import annotations

import numpy as np


def frequencies(rd, theta, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=0):
    """Radians a position of each of the rd / 2 pairs."""
    out = []
    for i in range(rd // 2):
        g = float(theta) ** (-2.0 * i / rd)
        if scaling == "none":
            out.append(g)
        elif scaling == "linear":
            out.append(g / factor)
        elif scaling == "base":
            out.append((theta * factor ** (rd / (rd - 2.0))) ** (-2.0 * i / rd))
        elif scaling == "wavelength":
            wavelength = 2 * np.pi / g
            if wavelength < original_len / high:
                out.append(g)
            elif wavelength > original_len / low:
                out.append(g / factor)
            else:
                s = (original_len / wavelength - low) / (high - low)
                out.append((1 - s) * g / factor + s * g)
        else:
            at = lambda turns: rd * np.log(original_len / (turns * 2 * np.pi)) / (2 * np.log(theta))  # noqa: E731
            first, last = max(np.floor(at(high)), 0), min(np.ceil(at(low)), rd - 1)
            s = min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
            out.append(g / factor * s + g * (1 - s))
    return np.array(out)


def turn(x, pos, freq, gain=None, eps=1e-6, layout="half", factor=1.0):
    """Row(s) x [..., d] at position `pos`."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    m = len(freq)
    a, b = (slice(0, m), slice(m, 2 * m)) if layout == "half" else (slice(0, 2 * m, 2), slice(1, 2 * m, 2))
    z = (x[..., a] + 1j * x[..., b]) * factor * np.exp(1j * (float(pos) * freq))
    y = x.copy()
    y[..., a], y[..., b] = z.real, z.imag
    return y
