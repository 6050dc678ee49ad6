"""Plain numpy definitions of the 8-bit forms of a block's input, in float64 (codes and scales as the C header states them)."""
import numpy as np

GROUP = 32
BOUNDS = {"bf16": (-126, 121), "f32": (-126, 121), "f16": (-24, 9)}


def pack(x, dtype):
    """(codes int8 [count], steps uint8 [ceil(count / 32)]) of a flat array of values of the storage type."""
    lo, hi = BOUNDS[dtype]
    x = np.asarray(x, np.float64).ravel()
    groups = -(-x.size // GROUP)
    v = np.zeros(groups * GROUP)
    v[:x.size] = x
    v = v.reshape(groups, GROUP)
    bad = ~np.isfinite(v).all(1)
    v = np.where(bad[:, None], 0.0, v)
    top = np.abs(v).max(1, initial=0.0)
    e = np.frexp(top)[1] - 7                               # top 2^-e in [64, 128), or 0
    e = np.where(np.rint(np.ldexp(top, -e)) > 127, e + 1, e)
    e = np.clip(np.where(top == 0, lo, e), lo, hi)
    q = np.clip(np.rint(np.ldexp(v, -e[:, None])), -127, 127)
    q = np.where(q == 0, np.sign(v), q)
    return q.astype(np.int8).ravel()[:x.size], np.where(bad, 255, e + 127).astype(np.uint8)


def unpack(codes, steps):
    steps = np.repeat(np.asarray(steps, np.int64), GROUP)[:codes.size]
    v = np.ldexp(codes.astype(np.float64), steps - 127)
    return np.where(steps == 255, np.nan, v)


def row_codes(x):
    """(codes, scale) of every row of a matrix of values of the storage type; the factor is 127 times the
    reciprocal, each rounded to fp32."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x).all(1)
    v = np.where(finite[:, None], x, 0.0)
    top = np.abs(v).max(1).astype(np.float32)
    live = finite & (top >= 2.0 ** -100)
    with np.errstate(divide="ignore", over="ignore"):
        inv = np.where(live, np.float32(127) * (np.float32(1) / np.where(live, top, np.float32(1))), np.float32(0)).astype(np.float64)
    scale = np.where(finite, np.where(live, top.astype(np.float64) / 127, 0.0), np.nan)
    return np.rint(v * inv[:, None]), scale


def deploy_forward(x, w, b, gamma, beta, mu_hat, var_hat, eps, add=None, relu=False):
    """z [rows, C_out] before any rounding, the size of its product term, and the weights' codes and scales."""
    xq, xs = row_codes(x)
    wq, wa = row_codes(w)
    s = gamma / np.sqrt(var_hat + eps)
    shift = ((b if b is not None else 0.0) - mu_hat) * s + beta
    product = (xq @ wq.T) * xs[:, None] * (wa * s)[None, :]
    z = product + shift
    out = z if add is None else z + add
    return {"z": np.maximum(out, 0.0) if relu else out, "before_add": z, "product": product, "w_codes": wq, "w_scale": wa * s,
            "b_fused": shift}
