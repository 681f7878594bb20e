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


def axes_frequencies(axes, theta, alternating=False, restart=False, blocks=1, **scaling):
    """Pair by pair of all blocks: angle from one position to the next and axis; and the factor on turned channels."""
    order, left, magnitude = [], list(axes), 1.0
    while sum(left):
        for a, n in enumerate(axes):
            take = (left[a] > 0) if alternating else left[a]
            order += [(a, n - left[a] + j) for j in range(take)]
            left[a] -= take
    out = []
    for i, (a, nth) in enumerate(order):
        r, place = (2 * axes[a], nth) if restart else (2 * sum(axes), i)
        f, magnitude = rotary_frequencies(r, theta, **scaling)
        out.append((f[place], a))
    return np.array([f for f, _ in out] * blocks), np.array([a for _, a in out] * blocks), magnitude


def rotary_by_axes(x, positions, turns, axis, magnitude, interleaved, blocks=1, inverse=False):
    """rotary() with positions [axes][tokens] and the axis of every pair, block of channels by block of channels."""
    x = np.asarray(x, np.float64)
    n = len(turns) // blocks
    out, size = x.copy(), np.zeros_like(x)
    for b in range(blocks):
        for j in range(n):
            i = b * n + j
            lo = 2 * n * b + (2 * j if interleaved else j)
            hi = lo + (1 if interleaved else n)
            angle = np.array([math.fmod(float(p) * turns[i], 1.0) * 2 * math.pi for p in positions[axis[i]]])[:, None]
            c, s = magnitude * np.cos(angle), magnitude * np.sin(-angle if inverse else angle)
            with np.errstate(invalid="ignore"):
                out[..., lo] = x[..., lo] * c - x[..., hi] * s
                out[..., hi] = x[..., hi] * c + x[..., lo] * s
                size[..., lo] = size[..., hi] = np.abs(x[..., lo]) + np.abs(x[..., hi])
    return out, size


def differential(q, k, v, scale, lam, norm=None, gain=1.0, half_step=0.0, least=0.0):
    """One request: q [H, 2, d], k and v [n, G, 2 d] (a head's keys are [K_1 | K_2]), lam [H]; norm: None or (eps, weight [2 d]).  All
    64 bits.  Returns out [H, 2 d] and how far a result may be off whose exponentials were rounded by half_step of themselves, or
    by `least` where they are smaller than that goes, whose products and sums ran in 32 bits, and which was rounded by half_step."""
    heads, _, d = q.shape
    n, group, u = len(k), heads // k.shape[1], 2.0 ** -24
    out, off = np.zeros((heads, 2 * d)), np.zeros((heads, 2 * d))
    for h in range(heads):
        o, e = [], []
        for m in range(2):
            keys, values = k[:, h // group, m * d:(m + 1) * d], v[:, h // group]
            x = scale * (keys @ q[h, m])
            p = np.exp(x - x.max())
            total = p.sum()
            p = p / total
            o.append(p @ values)
            away = np.abs(values - o[-1])
            # a weight is off by: its rounding, which the sum of weights shares; its score, d products summed in 32 bits, times
            # the scale and log2(e), less a reference; the exponential, 2 ulp; the rescalings of partial sums, a few more
            score = (d + 3) * u * scale * (np.abs(keys) @ np.abs(q[h, m])) + 4 * u * np.abs(x).max() + 16 * u
            weight = p * (half_step + score) + least / total
            # the sums of weights and of products run over n tokens in 32 bits
            e.append((weight @ away) / (1 - half_step - score.max()) + (2 * n + 32) * u * (p @ np.abs(values)))
        x = o[0] - lam[h] * o[1]
        dx = e[0] + abs(lam[h]) * e[1] + 2 * u * (np.abs(o[0]) + np.abs(lam[h] * o[1]))
        if norm is not None:
            eps, w = norm
            rho, drho = np.sqrt(np.mean(x * x) + eps), np.sqrt(np.mean(dx * dx))
            y = x / rho * w
            dx = np.abs(w) * (dx + np.abs(x) * drho / rho) / max(rho - drho, np.sqrt(eps)) + (2 * d + 8) * u * np.abs(y)
            x = y
        out[h], dx = gain * x, abs(gain) * dx
        off[h] = dx + half_step * (np.abs(out[h]) + dx) + 2 * u * np.abs(out[h]) + least
    return out, off


def block_table(page_size, page_off, page_ids, tokens, width):
    """Row by row: the pages that hold the tokens, -1 behind them."""
    rows = []
    for s, n in enumerate(tokens):
        begin, end = int(page_off[s]), int(page_off[s + 1])
        pages = []
        for i in range(min(-(-max(int(n), 0) // page_size), width)):
            if 0 <= begin and begin + i < min(end, len(page_ids)):
                pages.append(int(page_ids[begin + i]))
        rows.append(pages + [-1] * (width - len(pages)))
    return np.array(rows, np.int64).reshape(len(tokens), width)


def slot_map(page_size, num_pages, table, tokens, new, num_tokens, before=None, spare=None):
    """Token by token.  (positions, slots, sequences, offsets, tokens, taken, table)"""
    table = np.array(table, np.int64)
    width = table.shape[1]
    positions, slots, sequences, offsets, now, taken = [], [], [], [0], [], 0
    for s in range(len(tokens)):
        n = held = max(int(tokens[s]), 0)
        held = min(-(-held // page_size), width)        # pages that the table has
        for _ in range(max(int(new[s]), 0)):
            if len(slots) == num_tokens:
                break
            page = n // page_size
            if spare is not None and held <= page < width:
                i = int(spare[taken]) if taken < len(spare) else -1
                table[s, page] = i if 0 <= i < num_pages else -1
                held, taken = held + 1, taken + 1
            entry = int(table[s, page]) if page < width else -1
            slots.append(entry * page_size + n % page_size if 0 <= entry < num_pages else -1)
            positions.append(n + (0 if before is None else int(before[s])))
            sequences.append(s)
            n += 1
        offsets.append(len(slots))
        now.append(min(n, 2 ** 31 - 1))
    behind = num_tokens - len(slots)
    return (np.array(positions + [0] * behind, np.int64), np.array(slots + [-1] * behind, np.int64), np.array(sequences + [-1] * behind, np.int64),
            np.array(offsets), np.array(now, np.int64), np.array([taken]), table)


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
