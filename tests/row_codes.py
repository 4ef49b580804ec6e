"""Codes of rows against their definition, saturated ones included."""
import numpy as np


def off_from_definition(q, y, total, u, block):
    """How much farther than allowed each code is from its definition, clip(127 y / max|y| + u / 2, -127, 127), rounded to nearest (by half a
    step at most): where the kernel's fp32 arithmetic is granted what it may lose, a stage of the transform 2^-24 of the
    block's sum of magnitudes `total`, the factor 127 / max, the product with it and the addition of the dither 2^-24 of at most 128 each.
    Rows whose largest magnitude is 0 have codes 0."""
    most = np.abs(y).max(axis=1)
    live = most > 0
    rel = np.zeros_like(most)
    rel[live] = (block + 1) * total[live] / most[live] * 2.0 ** -24 + 4 * 2.0 ** -24
    want = np.zeros_like(y)
    want[live] = np.clip(127 * y[live] / most[live, None] + u[live] / 2, -127, 127)
    return np.abs(q - want) - (0.5 * live + 2 * 128 * rel)[:, None]
