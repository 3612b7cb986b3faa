"""CPU oracle (test infrastructure only): rotary positions in every pairing, over part of a head, at scaled frequencies.

A pair is a complex number and is multiplied by magnitude * exp(i * position * f).  All in fp64.
"""
import math

import numpy as np


def frequencies(rot, theta, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=0):
    """f_i = theta^(-2i/rot), i < rot/2, scaled:
    linear  f_i / factor (positions are interpolated);
    base    theta grows by factor^(rot/(rot-2)): the last pair, i = rot/2 - 1, slows by exactly factor, the first not at all;
    parts   pairs that make fewer than `low` turns within original_len positions are interpolated, those that make more than
            `high` are kept, and between the two the share of the kept frequency grows linearly with the turns."""
    out = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "base":
            if i:
                f *= factor ** (-i / (rot / 2 - 1))
        elif scaling == "parts":
            turns = original_len / (2 * math.pi / f)
            if turns <= low:
                f /= factor
            elif turns < high:
                kept = (turns - low) / (high - low)
                f = kept * f + (1 - kept) * (f / factor)
        elif scaling != "none":
            raise ValueError(scaling)
        out.append(f)
    return np.array(out)


def turn(x, positions, freq, interleaved=False, magnitude=1.0):
    """x [R, heads, d_h], positions [R]; the first 2 * len(freq) entries of a head turn, pairs (i, i + len(freq)) or (2i, 2i + 1)."""
    x = np.asarray(x, np.float64)
    n = len(freq)
    by = magnitude * np.exp(1j * np.asarray(positions, np.float64)[:, None] * freq[None, :])[:, None, :]
    out = x.copy()
    if interleaved:
        z = (x[..., 0:2 * n:2] + 1j * x[..., 1:2 * n:2]) * by
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = z.real, z.imag
    else:
        z = (x[..., :n] + 1j * x[..., n:2 * n]) * by
        out[..., :n], out[..., n:2 * n] = z.real, z.imag
    return out
