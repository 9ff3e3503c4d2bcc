"""Oracle: rotary positions in float64 (test infrastructure only).

Pair i of a row's first ``rot`` dims, (2i, 2i + 1) or (i, i + rot / 2), turns by
the angle p * freqs[i] at position p and is multiplied by m; the other dims are
as they were.  The backward pass is the transposed map, written out here as the
product with the transposed 2 x 2 matrix.
"""

import math

import numpy as np


def frequencies(rot, base=10000.0, scaling=None, factor=1.0, original_len=0):
    """(freqs, m): one pair at a time, from the definitions of the scalings."""
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2.0)) if scaling == "ntk" else base
        f = 1.0 / b ** (2.0 * i / rot)
        if scaling == "linear":
            f = f / factor
        if scaling == "yarn":
            wavelength = 2.0 * math.pi / f
            turns = original_len / wavelength
            if turns <= 1.0:
                f = f / factor
            elif turns < 32.0:
                w = (turns - 1.0) / (32.0 - 1.0)
                f = (1.0 - w) * (f / factor) + w * f
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def tree_positions(seq_len, parents_b):
    """Position of each node: the prefix length plus its number of ancestors."""
    out = []
    for n in range(len(parents_b)):
        depth, p = 0, int(parents_b[n])
        while p != -1:
            depth, p = depth + 1, int(parents_b[p])
        out.append(int(seq_len) + depth)
    return out


def rope(x, positions, freqs, m=1.0, interleaved=False, backward=False):
    """x [B, T, H, D] float64, positions [B, T] -> the turned rows."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    half = len(freqs)
    for i in range(half):
        d1, d2 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        a = np.asarray(positions, dtype=np.float64) * freqs[i]
        c, s = m * np.cos(a)[:, :, None], m * np.sin(a)[:, :, None]
        matrix = ((c, s), (-s, c)) if backward else ((c, -s), (s, c))
        y[..., d1] = matrix[0][0] * x[..., d1] + matrix[0][1] * x[..., d2]
        y[..., d2] = matrix[1][0] * x[..., d1] + matrix[1][1] * x[..., d2]
    return y
