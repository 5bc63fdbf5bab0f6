"""Norm of query / key heads with the rotation by position, and its gradient, in 64 bits: whole-array numpy written from the
definition (a rotation matrix per position, applied and transposed), for the tests."""
import numpy as np


def rotation(cos_sin, positions, D, adjacent):
    """[T, D, D]: z = M y."""
    T, rot = len(positions), cos_sin.shape[1]
    M = np.zeros((T, D, D))
    M[:, np.arange(D), np.arange(D)] = 1.0
    h = rot // 2
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + h)
        c, s = cos_sin[positions, i], cos_sin[positions, h + i]
        M[:, a, a], M[:, a, b], M[:, b, b], M[:, b, a] = c, -s, c, s
    return M


def forward(x, w, M, eps):
    """x [T, H, D] -> z, and the sums of the magnitudes that are added up in z."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    y = x * r * w
    return np.matmul(y, M.transpose(0, 2, 1)), np.matmul(np.abs(y), np.abs(M).transpose(0, 2, 1))


def backward(dz, x, w, M, eps):
    """dx, dw, and for each the sums of magnitudes."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dy, dy_abs = np.matmul(dz, M), np.matmul(np.abs(dz), np.abs(M))
    g, g_abs = dy * w, dy_abs * np.abs(w)
    dx = r * (g - n * (g * n).mean(-1, keepdims=True))
    dx_abs = r * (g_abs + np.abs(n) * (g_abs * np.abs(n)).mean(-1, keepdims=True))
    return dx, (dy * n).sum((0, 1)), dx_abs, (dy_abs * np.abs(n)).sum((0, 1))


def table(max_positions, rot):
    angle = np.arange(max_positions)[:, None] * 10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
