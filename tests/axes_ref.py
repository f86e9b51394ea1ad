"""Plain 64-bit forms of the norm and rotation of heads by positions of several axes, on the CPU."""
import numpy as np


def angles(positions, axis, freq):
    """[T, rot / 2]: position of each pair's axis times its frequency.  positions [axes, T]."""
    return np.asarray(positions, np.float64)[np.asarray(axis)].T * np.asarray(freq, np.float64)


def rotate(y, angle, interleaved):
    """y [T, h, d], its first pairs turned by angle [T, pairs]: as complex numbers times e^(i angle)."""
    y, n = np.array(y, np.float64), angle.shape[1]
    if n == 0:
        return y
    i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    z = (y[..., i] + 1j * y[..., j]) * np.exp(1j * angle)[:, None]
    y[..., i], y[..., j] = z.real, z.imag
    return y


def heads(x, w, angle, eps, interleaved):
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return rotate(x, angle, interleaved)


def heads_backward(dy, x, w, angle, eps, interleaved):
    """(gradient of x, gradient of w)."""
    x, g = np.asarray(x, np.float64), rotate(dy, -angle, interleaved)
    if w is None:
        return g, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, h = x * r, g * w
    return r * (h - xh * (h * xh).mean(-1, keepdims=True)), (g * xh).sum((0, 1))
