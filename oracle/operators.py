"""Plain 64-bit implementations of the operators around a decode step.  TEST INFRASTRUCTURE ONLY."""
from __future__ import annotations

import math

import numpy as np


def rotary_frequencies(r, theta, kind=None, factor=1.0, original_length=0, low=1.0, high=4.0, fast=32.0, slow=1.0):
    """Angle of every pair from one position to the next, pair by pair, and the factor on turned channels."""
    out, magnitude = [], 1.0
    for i in range(r // 2):
        base = theta * factor ** (r / (r - 2)) if kind == "ntk" and r > 2 else theta
        f = base ** (-(2 * i) / r)
        if kind == "linear":
            f = f / factor
        if kind == "wavelength":
            length = 2 * math.pi / f                    # positions of a whole turn
            if length > original_length / low:
                f = f / factor
            elif length > original_length / high:
                smooth = (original_length / length - low) / (high - low)
                f = (1 - smooth) * f / factor + smooth * f
        if kind == "yarn":
            def pair(turns):
                return r * math.log(original_length / (turns * 2 * math.pi)) / (2 * math.log(theta))
            a, b = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), r - 1)
            ramp = min(max((i - a) / (b - a if b > a else 0.001), 0.0), 1.0)
            f = f / factor * ramp + f * (1 - ramp)
            magnitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
        out.append(f)
    return np.array(out), magnitude


def rotary(x, positions, turns, magnitude, interleaved, inverse=False):
    """x [tokens, heads, d] float64, every pair of channels turned as a complex number, pair i by turns[i] whole turns a
    position; and |a| + |b| of the pair behind every channel (0 where it passes), which the rounding errors go by."""
    x = np.asarray(x, np.float64)
    r = 2 * len(turns)
    first = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
    second = first + 1 if interleaved else first + r // 2
    out, size = x.copy(), np.zeros_like(x)
    for t, n in enumerate(positions):
        turn = magnitude * np.exp((-1j if inverse else 1j) * np.fmod(float(n) * turns, 1.0) * 2 * math.pi)
        with np.errstate(invalid="ignore"):
            out[t][:, first] = x[t][:, first] * turn.real - x[t][:, second] * turn.imag
            out[t][:, second] = x[t][:, second] * turn.real + x[t][:, first] * turn.imag
            size[t][:, first] = size[t][:, second] = np.abs(x[t][:, first]) + np.abs(x[t][:, second])
    return out, size
