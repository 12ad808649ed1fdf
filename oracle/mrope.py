"""Oracle rotary positions on three axes (time, height, width).

TEST INFRASTRUCTURE ONLY (see the package docstring).

Positions of a segment, token by token: a counter n starts at 0; a prompt or
text token stands at (n, n, n) and n grows by one; the patch (f, y, x) of a
screenshot of t frames of h x w patches that opens at n stands at (n + e f,
n + y, n + x), e its time step, and behind the screenshot n is one more than
the largest position that it used.

Rotation: the pair (i, i + d/2) of a head turns by pos[axis(i)] base^(-2i/d);
the first pairs are on the time axis, the next on the height, the last on the
width.
"""
from __future__ import annotations

import numpy as np

IMAGE = 1


def segment_positions(kind, step, grid_of):
    """kind, step: of each token of one segment; grid_of(turn) = (t, h, w, e).
    Returns [3, length]."""
    out = np.zeros((3, len(kind)), np.int64)
    n, i = 0, 0
    while i < len(kind):
        if kind[i] != IMAGE:
            out[:, i] = n
            n += 1
            i += 1
            continue
        t, h, w, e = (int(v) for v in grid_of(int(step[i])))
        top = n
        for f in range(t):
            for y in range(h):
                for x in range(w):
                    assert kind[i] == IMAGE
                    out[:, i] = (n + e * f, n + y, n + x)
                    top = max(top, n + e * f, n + y, n + x)
                    i += 1
        n = top + 1
    return out


def positions(layout, spans, grid, packed):
    """[3, packed] positions of every packed row (-1 in padding); grid [num_steps, 4]."""
    out = np.full((3, packed), -1, np.int64)
    for sg in layout.segments:
        s0 = int(spans.step_offsets[sg.traj])
        out[:, sg.start:sg.start + sg.length] = segment_positions(
            sg.kind, sg.step, lambda turn, s0=s0: grid[s0 + turn - 1])
    return out


def angles(pos, d, sections, base):
    """[rows, d/2] angles of pos [3, rows]."""
    axis = np.repeat(np.arange(3), sections)
    assert len(axis) == d // 2
    inv = np.float64(base) ** (-2.0 * np.arange(d // 2) / d)
    return np.asarray(pos, np.float64)[axis].T * inv


def rotate(x, pos, sections, base, inverse=False):
    """x [rows, heads, d] rotated; rows with a negative position are copied
    (inverse: the transpose, zeros there)."""
    d = x.shape[-1]
    t = angles(np.maximum(pos, 0), d, sections, base)[:, None]
    c, s = np.cos(t), np.sin(t) * (-1.0 if inverse else 1.0)
    a, b = x[..., :d // 2], x[..., d // 2:]
    y = np.concatenate([a * c - b * s, b * c + a * s], -1)
    pad = (np.asarray(pos) < 0).any(0)
    y[pad] = 0.0 if inverse else x[pad]
    return y
