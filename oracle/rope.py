"""Head norms and position rotation in extended precision (numpy long double): the definition that the rotation
kernels are held to."""
import numpy as np

L = np.longdouble


def norm(x, weight, eps):
    """x [..., D] / sqrt(mean(x^2) + eps) * weight; weight None: x."""
    x = np.asarray(x, dtype=L)
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + L(np.float32(eps))) * np.asarray(weight, dtype=L)


def angles(positions, inv_freq, axis=None):
    """Angles [tokens, pairs] of positions [axes, tokens]."""
    positions = np.asarray(positions, dtype=L)
    axis = np.zeros(len(inv_freq), dtype=int) if axis is None else np.asarray(axis, dtype=int)
    return positions[axis].T * np.asarray(inv_freq, dtype=L)


def partners(d, pairs, interleaved):
    """For every value of a row: its pair, its partner, and the sign of the sine in its own sum."""
    pair, mate, sign = np.full(d, -1), np.arange(d), np.zeros(d)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        pair[a] = pair[b] = i
        mate[a], mate[b] = b, a
        sign[a], sign[b] = -1, 1
    return pair, mate, sign


def rotate(y, ang, interleaved, scale):
    """Rows y [tokens, H, D] turned by ang [tokens, pairs]."""
    y = np.asarray(y, dtype=L)
    pair, mate, sign = partners(y.shape[-1], ang.shape[1], interleaved)
    on = pair >= 0
    scale = L(np.float32(scale))
    c = np.where(on, np.cos(ang)[:, pair] * scale, 1)[:, None]
    s = np.where(on, np.sin(ang)[:, pair] * scale, 0)[:, None] * sign
    return y * c + y[..., mate] * s
