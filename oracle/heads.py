"""CPU fp64 oracle of what stands between the projection and the reader: norm of query and key heads, rotary embedding in both
layouts and of part of a head, their gradients, and tables scaled for long contexts.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py): imported by tests/ alone; the GPU library shares no code with it.

The paper is silent on all of it (Sec. 2.1 speaks of query, key and value vectors only); the formulas are the textbook ones.
Pinned by tests/test_heads_pins.py.  Every function also returns or takes what a tolerance needs: the size of what was added up.
"""
from __future__ import annotations

import numpy as np


def _pairs(rot: int, interleaved: bool):
    """Indexes of the first and second features of the turned pairs."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, cos, sin, interleaved: bool, size: bool = False) -> np.ndarray:
    """x [rows, heads, d]; cos, sin [rows, pairs].  size: magnitudes are added instead (what the rounding of a sum is relative to)."""
    x = np.asarray(x, np.float64)
    out = np.abs(x) if size else x.copy()
    a, b = _pairs(2 * cos.shape[1], interleaved)
    c, s = np.asarray(cos, np.float64)[:, None, :], np.asarray(sin, np.float64)[:, None, :]
    if size:
        out[..., a] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
        out[..., b] = np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    else:
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def normed(x, w, eps: float) -> np.ndarray:
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)


def heads(x, w, eps, cos, sin, interleaved):
    """(result, size): w None: no norm; cos None: no rotation."""
    y = np.asarray(x, np.float64) if w is None else normed(x, w, eps)
    if cos is None:
        return y, np.abs(y)
    return turn(y, cos, sin, interleaved), turn(y, cos, sin, interleaved, size=True)


def heads_back(x, g_out, w, eps, cos, sin, interleaved):
    """(dx, its size, dw, its size) from the gradient of the result."""
    g_out = np.asarray(g_out, np.float64)
    g, gs = g_out, np.abs(g_out)
    if cos is not None:
        g, gs = turn(g_out, cos, -np.asarray(sin, np.float64), interleaved), turn(g_out, cos, sin, interleaved, size=True)
    if w is None:
        return g, gs, None, None
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, us = g * w, gs * np.abs(w)
    dx = r * u - x * r ** 3 * (u * x).mean(-1, keepdims=True)
    dxs = r * us + np.abs(x) * r ** 3 * (us * np.abs(x)).mean(-1, keepdims=True)
    return dx, dxs, (g * x * r).sum((0, 1)), (gs * np.abs(x) * r).sum((0, 1))


def tables(rot, base, first, rows, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0, magnitude=1.0):
    """cos, sin [rows, rot / 2] in extended precision."""
    f = np.longdouble
    pi = f("3.14159265358979323846264338327950288")
    i = np.arange(rot // 2).astype(f)
    theta = np.exp(-i * 2 / f(rot) * np.log(f(base)))
    if scaling == "linear":
        theta = theta / f(factor)
    elif scaling == "by_parts":
        out = []
        for t in theta:
            turns = f(original) * t / (2 * pi)
            if turns >= high:
                out.append(t)
            elif turns <= low:
                out.append(t / f(factor))
            else:
                g = (turns - f(low)) / (f(high) - f(low))
                out.append(g * t + (1 - g) * t / f(factor))
        theta = np.array(out)
    angle = np.arange(first, first + rows).astype(f)[:, None] * theta[None, :]
    return np.cos(angle) * f(magnitude), np.sin(angle) * f(magnitude)
