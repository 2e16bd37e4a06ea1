"""Rotary positions of several axes on a qkv matrix, in 64 bits, from the definitions: pair p of a head's query and key turns by
positions[axis of p][row] * scale[axis of p] * frequency of p."""
import math

import numpy as np


def ladder(pairs, base=10000.0, in_turn=False, shared=False):
    """[(axis, frequency)] of every pair."""
    order = []
    if in_turn:
        left = list(pairs)
        while sum(left):
            for a, k in enumerate(left):
                if k:
                    order.append(a)
                    left[a] -= 1
    else:
        for a, k in enumerate(pairs):
            order += [a] * k
    out, seen = [], {}
    for p, a in enumerate(order):
        k = seen.get(a, 0)
        seen[a] = k + 1
        out.append((a, base ** -(p / len(order) if shared else k / pairs[a])))
    return out


def rotate(qkv, positions, n, pairs, *, scale=None, base=10000.0, interleaved=False, in_turn=False, shared=False, back=False):
    """qkv [rows, 3h] with columns head-major (head, {Q, K, V}, d); positions [axes, rows].  Returns [rows, 3h] in 64 bits."""
    x = np.array(qkv, dtype=np.float64)
    rows = x.shape[0]
    heads = x.reshape(rows, n, 3, -1)
    P = sum(pairs)
    for p, (axis, freq) in enumerate(ladder(pairs, base, in_turn, shared)):
        angle = [math.fmod(float(t) * (1.0 if scale is None else scale[axis]) * freq, 2 * math.pi) for t in positions[axis]]
        c, s = np.cos(angle)[:, None, None], (-1 if back else 1) * np.sin(angle)[:, None, None]
        e, f = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
        u, v = heads[:, :, :2, e].copy(), heads[:, :, :2, f].copy()
        heads[:, :, :2, e] = u * c - v * s
        heads[:, :, :2, f] = u * s + v * c
    return x
