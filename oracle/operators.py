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


class Pages:
    """Who holds which page: lists of holders, nothing clever."""

    def __init__(self, n):
        self.holders = [0] * n

    def free(self):
        return [p for p, h in enumerate(self.holders) if h == 0]

    def take(self, n):
        ids = self.free()[:n]
        assert len(ids) == n
        for p in ids:
            self.holders[p] = 1
        return ids

    def fork(self, page_size, lists, tokens, parents):
        """New lists of the sequences that go on from `parents`, and the runs to copy."""
        free, out, runs = self.free(), [], []
        gone_on = set()
        for s in parents:
            whole = tokens[s] // page_size
            mine = list(lists[s])
            alone = all(self.holders[p] == 1 for p in mine[whole:])
            if not alone or s in gone_on:
                for i in range(whole, len(mine)):
                    page = free.pop(0)
                    if i == whole and tokens[s] % page_size:
                        runs.append((mine[i], 0, page, 0, tokens[s] % page_size))
                    mine[i] = page
            gone_on.add(s)
            out.append(mine)
        for p in (p for pages in out for p in pages):
            self.holders[p] += 1
        for p in (p for pages in lists for p in pages):
            self.holders[p] -= 1
        assert min(self.holders) >= 0
        return out, runs

    def compact(self, page_size):
        n = sum(h != 0 for h in self.holders)
        high = [p for p, h in enumerate(self.holders) if h and p >= n]
        low = [p for p in self.free() if p < n]
        for a, b in zip(high, low):
            self.holders[b], self.holders[a] = self.holders[a], 0
        return [(a, 0, b, 0, page_size) for a, b in zip(high, low)]


def beam_scores(logits, scores, finished=None, eos=0):
    """Score of every continuation [batch, beams, vocab], float64."""
    x = np.array(logits, np.float64)
    x[np.isnan(x)] = -np.inf
    x[x == np.inf] = float(np.finfo(np.float32).max)
    c = np.array(scores, np.float64)
    c[np.isnan(c) | (c == np.inf)] = -np.inf
    top = x.max(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        y = (x - top) - np.log(np.exp(x - top).sum(-1, keepdims=True))
    y[np.isnan(y)] = -np.inf
    if finished is not None:
        done = np.asarray(finished) != 0
        y[done] = -np.inf
        y[done, eos] = 0.0
    return c[..., None] + y


def beam_select(logits, scores, k, finished=None, eos=0):
    """(scores, beams, tokens), each [batch, k]: the best continuations, equal ones by the lowest beam and token."""
    s = beam_scores(logits, scores, finished, eos)
    flat = s.reshape(len(s), -1)
    order = np.argsort(-flat, axis=1, kind="stable")[:, :k]
    return np.take_along_axis(flat, order, 1), order // s.shape[2], order % s.shape[2]
