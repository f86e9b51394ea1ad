"""Plain 64-bit forms of residual and norm, on the CPU."""
import numpy as np


def norm(s, w, eps):
    s = np.asarray(s, np.float64)
    y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    return y if w is None else y * w


def norm_backward(dy, s, w, dsum, eps):
    """(gradient of the sum, gradient of w)."""
    s, g = np.asarray(s, np.float64), np.asarray(dy, np.float64)
    r = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    u, h = s * r, g if w is None else g * w
    gx = r * (h - u * (h * u).mean(-1, keepdims=True))
    return gx if dsum is None else gx + dsum, (g * u).sum(0)


def scales(y, group=128):
    """Largest magnitude of each group of channels / 448."""
    T, D = y.shape
    return np.abs(y).reshape(T, D // group, group).max(-1, initial=0.0) / 448
