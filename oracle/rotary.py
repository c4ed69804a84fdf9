"""Rotary positions in float64, one row, head and pair at a time."""

import math

import numpy as np


def turns(dim, theta, scaling="plain", factor=1.0, trained=0.0, fast=0.0, slow=0.0):
    """Turns a position of each pair (no 2 pi in a frequency's name: f radians)."""
    out = []
    for i in range(dim // 2):
        f = math.exp(-math.log(theta) * 2 * i / dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "base" and dim > 2:
            stretched = theta * factor ** (dim / (dim - 2))
            f = stretched ** (-2 * i / dim)
        elif scaling == "ramp":
            r = trained * f / (2 * math.pi)
            if r <= slow:
                f = f / factor
            elif r < fast:
                w = (r - slow) / (fast - slow)
                f = f * w + f / factor * (1 - w)
        out.append(f / (2 * math.pi))
    return out


def rotate(x, dim, pos, per, pairs=False, gain=1.0, inverse=False):
    """x [rows, heads, width], the first `dim` elements turned by pos * per turns."""
    y = np.array(x, np.float64)
    for r in range(len(y)):
        for i in range(dim // 2):
            whole = float(pos[r]) * per[i]
            t = 2 * math.pi * (whole - round(whole)) * (-1 if inverse else 1)
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + dim // 2)
            u, v = y[r, :, a].copy(), y[r, :, b].copy()
            y[r, :, a] = gain * (u * math.cos(t) - v * math.sin(t))
            y[r, :, b] = gain * (v * math.cos(t) + u * math.sin(t))
    return y
