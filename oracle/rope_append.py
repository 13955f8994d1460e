"""Oracle of norms and rotations in 64 bits, with complex numbers."""
import numpy as np


def rms(x, w, eps):
    x = np.asarray(x, np.float64)
    if w is None:
        return x
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(w, np.float64)


def rotate(x, positions, inv_freq, axis=None, interleaved=False):
    """x [N, heads, D]; positions [axes, N]; the first 2 * len(inv_freq) elements turn."""
    x = np.array(x, np.float64)
    f = np.asarray(inv_freq, np.float64)
    half = f.size
    if half == 0:
        return x
    ax = np.zeros(half, int) if axis is None else np.clip(np.asarray(axis), 0, len(positions) - 1)
    ang = np.asarray(positions, np.float64)[ax].T * f
    z = x[..., 0:2 * half:2] + 1j * x[..., 1:2 * half:2] if interleaved else x[..., :half] + 1j * x[..., half:2 * half]
    z = z * np.exp(1j * ang)[:, None]
    if interleaved:
        x[..., 0:2 * half:2], x[..., 1:2 * half:2] = z.real, z.imag
    else:
        x[..., :half], x[..., half:2 * half] = z.real, z.imag
    return x
