"""The paged KV cache in float64 numpy, sequence by sequence and slot by slot.

Written from the definitions in include/dv.h: here a sequence is a list of pages, and a
pool holds its numbers per (layer, page, head, slot), values in slot order.
"""
from __future__ import annotations

import math

import numpy as np

PLAIN, LINEAR, TURNS, LOG_TURNS = range(4)


def frequencies(rot, base=10000.0, scaling=PLAIN, factor=1.0, low=1.0, high=4.0, ctx=1):
    """Radians per position of each of rot / 2 pairs."""
    out = []
    for i in range(rot // 2):
        f = 1.0 / base ** (2 * i / rot)
        if scaling == LINEAR:
            f /= factor
        elif scaling in (TURNS, LOG_TURNS):
            g = (lambda x: x) if scaling == TURNS else math.log
            turns = ctx / (2 * math.pi / f)
            stays = min(max((g(turns) - g(low)) / (g(high) - g(low)), 0.0), 1.0)
            f = stays * f + (1 - stays) * f / factor
        out.append(f)
    return np.array(out)


def turned(x, position, freq, interleaved, magnitude=1.0):
    """x [..., head_dim] at one position, as products of complex numbers."""
    y, n = np.array(x, dtype=np.float64), len(freq)
    a, b = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    z = (y[..., a] + 1j * y[..., b]) * magnitude * np.exp(1j * (position * freq))
    y[..., a], y[..., b] = z.real, z.imag
    return y


class Paged:
    def __init__(self, k, v, mass, page):
        """k, v [layers][pages][heads][page][head_dim], mass [layers][pages][heads][page]."""
        self.page = page
        self.k, self.v = np.array(k, dtype=np.float64), np.array(v, dtype=np.float64)
        self.mass = np.array(mass, dtype=np.float64)

    def places(self, pages, slots):
        """(page, place) of slots of a sequence; None for a page that is not in the pool."""
        out = []
        for x in slots:
            p = pages[x // self.page]
            out.append((p, x % self.page) if 0 <= p < self.k.shape[1] else None)
        return out

    def append(self, layer, pages, length, k, v):
        """Rows k, v [n][heads][head_dim], already turned."""
        for i, at in enumerate(self.places(pages, range(length, length + len(k)))):
            if at:
                self.k[layer, at[0], :, at[1]], self.v[layer, at[0], :, at[1]] = k[i], v[i]
                self.mass[layer, at[0], :, at[1]] = 0

    def gathered(self, x, layer, pages, n):
        """Slots 0..n of a sequence, [n][heads][..], and which of them are there."""
        at = self.places(pages, range(n))
        there = np.array([p is not None for p in at], dtype=bool)
        out = np.zeros((n, x.shape[2]) + x.shape[4:])
        for j, p in enumerate(at):
            if p is not None:
                out[j] = x[layer, p[0], :, p[1]]
        return out, there

    def scores(self, layer, pages, length, q, masks, scale, cap=0.0):
        """One sequence: z [n][query heads][slots], -inf where a row does not see.
        q [n][query heads][head_dim]; masks: per row a set of new rows."""
        n, heads = q.shape[:2]
        k, there = self.gathered(self.k, layer, pages, length + n)
        k = np.repeat(k, heads // k.shape[1], axis=1)
        z = np.full((n, heads, length + n), -np.inf)
        for i in range(n):
            see = np.array([there[j] and (j < length or j - length in masks[i]) for j in range(length + n)], dtype=bool)
            z[i][:, see] = scale * (q[i][:, None] * k[see].transpose(1, 0, 2)).sum(axis=2)
            if cap:
                z[i][:, see] = cap * np.tanh(z[i][:, see] / cap)
        return z

    def attention(self, layer, pages, length, q, masks, scale, cap=0.0):
        """out [n][query heads][head_dim], largest score and sum [n][query heads]."""
        z = self.scores(layer, pages, length, q, masks, scale, cap)
        v, _ = self.gathered(self.v, layer, pages, z.shape[2])
        group = q.shape[1] // v.shape[1]
        out, top, total = np.zeros(q.shape), np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
        for i in range(q.shape[0]):
            for h in range(q.shape[1]):
                see = z[i, h] != -np.inf
                if see.any():
                    top[i, h] = z[i, h, see].max()
                    w = np.exp(z[i, h, see] - top[i, h])
                    total[i, h] = w.sum()
                    out[i, h] = (w / total[i, h]) @ v[see, h // group]
        return out, top, total

    def add_mass(self, layer, pages, length, q, masks, scale, cap, counted, stats=None):
        """stats [n][query heads][2], or None: the attention's own."""
        z = self.scores(layer, pages, length, q, masks, scale, cap)
        if stats is None:
            _, top, total = self.attention(layer, pages, length, q, masks, scale, cap)
            stats = np.stack([top, total], axis=-1)
        group = q.shape[1] // self.k.shape[2]
        for i in range(q.shape[0]):
            for h in range(q.shape[1]):
                if counted >> i & 1:
                    for j in np.nonzero(z[i, h] != -np.inf)[0]:
                        page, at = pages[j // self.page], j % self.page
                        self.mass[layer, page, h // group, at] += np.exp(z[i, h, j] - stats[i, h, 0]) / stats[i, h, 1]

    def _move(self, layer, head, pages, pairs):
        """Slots (from, to) of a head, all at once."""
        got = []
        for come, to in pairs:
            (a,), (b,) = self.places(pages, [come]), self.places(pages, [to])
            if a and b:
                got.append((b, self.k[layer, a[0], head, a[1]].copy(), self.v[layer, a[0], head, a[1]].copy(),
                            self.mass[layer, a[0], head, a[1]]))
        for b, k, v, m in got:
            self.k[layer, b[0], head, b[1]], self.v[layer, b[0], head, b[1]], self.mass[layer, b[0], head, b[1]] = k, v, m

    def commit(self, pages, length, path):
        for layer in range(self.k.shape[0]):
            for head in range(self.k.shape[2]):
                self._move(layer, head, pages, [(length + p, length + i) for i, p in enumerate(path)])
        return length + len(path)

    def kept(self, layer, head, pages, length, budget, recent):
        """Slots that an eviction leaves, by counting for each slot those that come before it."""
        at = self.places(pages, range(length - recent))
        m = [(-1, 0.0) if p is None else (1, 0.0) if np.isnan(self.mass[layer, p[0], head, p[1]])
             else (0, float(self.mass[layer, p[0], head, p[1]])) for p in at]
        order = sorted(range(len(m)), key=lambda j: (-m[j][0], -m[j][1], j))
        return sorted(order[:budget - recent]) + list(range(length - recent, length))

    def evict(self, pages, length, budget, recent):
        if length <= budget:
            return length
        for layer in range(self.k.shape[0]):
            for head in range(self.k.shape[2]):
                kept = self.kept(layer, head, pages, length, budget, recent)
                self._move(layer, head, pages, list(zip(kept, range(budget))))
        return budget
