"""The layers of sequence models on plain arrays in fp64, [batch][channels][height][width]."""
import numpy as np


def shared_gates(a, channels, c_inner=1):
    """Gates [B][Cg][H][T] as each of `channels` channels sees them: ciphertext j of a gate serves m neighbouring ciphertexts."""
    m = channels // a.shape[1]
    return a[:, [(c // (m * c_inner)) * c_inner + c % c_inner for c in range(channels)]]


def recurrence(a, x, reverse=False, c_inner=1):
    a, h = shared_gates(a, x.shape[1], c_inner), x.copy()
    order = list(range(x.shape[3]))[::-1 if reverse else 1]
    for before, t in zip(order, order[1:]):
        h[..., t] += a[..., t] * h[..., before]
    return h


def recurrence_grad(a, h, g, reverse=False, c_inner=1):
    """(dx, da): da is zero at the token without a predecessor."""
    full = shared_gates(a, g.shape[1], c_inner)
    dx, da = g.copy(), np.zeros_like(g)
    order = list(range(g.shape[3]))[::-1 if reverse else 1]
    for before, t in list(zip(order, order[1:]))[::-1]:
        da[..., t] = dx[..., t] * h[..., before]
        dx[..., before] += full[..., t] * dx[..., t]
    out, m = np.zeros_like(a), g.shape[1] // a.shape[1]
    for c in range(g.shape[1]):
        out[:, (c // (m * c_inner)) * c_inner + c % c_inner] += da[:, c]
    return dx, out


def group_norm(x, gamma, beta, groups, eps, act_ratio=None):
    v = x.reshape(x.shape[0], groups, -1)
    v = (v - v.mean(-1, keepdims=True)) / np.sqrt(v.var(-1, keepdims=True) + eps)
    y = v.reshape(x.shape) * gamma[:, None, None] + beta[:, None, None]
    return y if act_ratio is None else y * y + act_ratio * y


def cubic_error(lo, hi, iterations):
    """The largest relative error of 1 / sqrt on [lo, hi] after the first line and that many odd cubics."""
    a, b = np.sqrt(lo / hi), 1.0
    for _ in range(iterations + 1):
        s, low = a * a + a * b + b * b, a * b * (a + b)
        c3 = 2.0 / (2.0 / 3.0 * s * np.sqrt(s / 3.0) + low)
        a, b = c3 * low, 2.0 - c3 * low
    return 1.0 - a


def noise(log_n, special, scale):
    """One standard deviation of a slot behind a division: residues rounded (variance 1/12 per coefficient and conversion source,
    special + 2 of them) in both polynomials, the second times a ternary secret of 2/3 N non-zeros: N sqrt((special + 2) / 18)."""
    return 2.0 ** log_n * np.sqrt((special + 2) / 18.0) / scale
