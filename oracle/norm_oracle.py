"""Group norm with an activation from its definition, in fp64 numpy, channels last.  Test infrastructure only."""
import numpy as np


def _act(y, act):
    if act == "relu":
        return np.where(y > 0, y, 0.0)
    if act == "silu":
        return y / (1.0 + np.exp(-y))
    return y


def _act_slope(y, act):
    if act == "relu":
        return (y > 0).astype(np.float64)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-y))
        return s + y * s * (1.0 - s)
    return np.ones_like(y)


def _act_slope_size(y, act):
    """SiLU's slope is a sum s + y s (1 - s) that vanishes near y = -1.28 while each term is rounded relative to itself: the sum of the
    terms' magnitudes."""
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-y))
        return s + np.abs(y) * s * (1.0 - s)
    return _act_slope(y, act)


def forward(x, groups, gamma, beta, eps, act):
    """x [n][h][w][c] -> z, mean [n][groups], rstd [n][groups]"""
    x = np.asarray(x, np.float64)
    n, h, w, c = x.shape
    v = x.reshape(n, h * w, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(var + eps)
    xhat = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    return _act(xhat * gamma + beta, act), mean, rstd


def backward(dz, x, groups, gamma, beta, mean, rstd, act):
    """dx, dgamma, dbeta, and the sums of magnitudes behind each: what rounding is measured against."""
    x, dz = np.asarray(x, np.float64), np.asarray(dz, np.float64)
    n, h, w, c = x.shape
    grouped = lambda t: t.reshape(n, h * w, groups, c // groups)
    wide = lambda t: np.broadcast_to(t[:, None, :, None], (n, h * w, groups, c // groups)).reshape(x.shape)
    mean, rstd = np.asarray(mean, np.float64), np.asarray(rstd, np.float64)
    m, r = wide(mean), wide(rstd)
    xhat = (x - m) * r
    dy = dz * _act_slope(xhat * gamma + beta, act)
    g = dy * gamma
    first, second = grouped(g).mean(axis=(1, 3)), grouped(g * xhat).mean(axis=(1, 3))
    dx = r * (g - wide(first) - xhat * wide(second))
    sized = np.abs(dz) * _act_slope_size(xhat * gamma + beta, act)
    gs = sized * np.abs(gamma)
    size = r * (gs + wide(grouped(gs).mean(axis=(1, 3))) + np.abs(xhat) * wide(grouped(gs * np.abs(xhat)).mean(axis=(1, 3))))
    over = (0, 1, 2)
    return dict(dx=dx, dgamma=(dy * xhat).sum(over), dbeta=dy.sum(over), dx_size=size, dgamma_size=(sized * np.abs(xhat)).sum(over),
                dbeta_size=sized.sum(over))
