"""Front end of an exact layer (norm of a head's row, rotary positions) in fp64 from the definitions in include/kvm.h (numpy only)."""
import numpy as np

U = 2.0 ** -24   # half a step of fp32, relative


def frequencies(r, base=10000.0, scaling="none", factor=1.0, original_len=0, low=1.0, high=32.0):
    """Radians per position of each pair, in extended precision."""
    w = np.longdouble(base) ** (-np.arange(0, r, 2, dtype=np.longdouble) / np.longdouble(max(r, 1)))
    if scaling == "linear":
        return w / np.longdouble(factor)
    if scaling == "parts":
        g = np.clip((original_len * w / (2 * np.longdouble(np.pi)) - low) / (high - low), 0, 1)
        return g * w + (1 - g) * w / np.longdouble(factor)
    return w


def pairs(r, layout):
    i = np.arange(r // 2)
    return (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)


def front(x, pos, norm="layer", eps=1e-5, rope_dims=0, layout="half", magnitude=1.0, weight=None, bias=None, **rope):
    """x [n, d] at positions pos [n], one head: (result [n, d], bound on what fp32 leaves of it [n, d]).

    The bound counts roundings of fp32 (u = 2^-24 each): the mean 12 of the largest |x|, the difference to it 2; the variance twice the relative error
    of what is squared, and 14 for its sum; the root 4 (2 ulp), the product with it, the weight and the bias 3; sin and cos 3 each (2 ulp and the
    argument's), 2^-50 of the angle for the way it is represented, the rotation 3."""
    x, d = np.asarray(x, np.float64), np.asarray(x).shape[1]
    err = np.zeros_like(x)
    if norm != "none":
        top = np.abs(x).max(1, keepdims=True)
        c = x - x.mean(1, keepdims=True) if norm == "layer" else x
        e_c = 16 * U * top if norm == "layer" else 0.0 * top
        sigma = np.sqrt((c * c).mean(1, keepdims=True) + eps)
        h = c / sigma
        err = e_c / sigma * (1 + np.abs(h)) + np.abs(h) * 14 * U
        w = 1.0 if weight is None else np.asarray(weight, np.float64)[None]
        b = 0.0 if bias is None else np.asarray(bias, np.float64)[None]
        x = h * w + b
        err = err * np.abs(w) + 2 * U * np.abs(x)
    if rope_dims:
        u, v = pairs(rope_dims, layout)
        angle = np.asarray(pos, np.longdouble)[:, None] * frequencies(rope_dims, **rope)[None]
        c, s = np.cos(angle).astype(np.float64) * magnitude, np.sin(angle).astype(np.float64) * magnitude
        off = magnitude * (6 * U + 2.0 ** -50 * angle.astype(np.float64))
        y, e = x.copy(), err.copy()
        y[:, u], y[:, v] = x[:, u] * c - x[:, v] * s, x[:, v] * c + x[:, u] * s
        e[:, u] = e[:, v] = magnitude * (err[:, u] + err[:, v]) + (off + 3 * U * magnitude) * (np.abs(x[:, u]) + np.abs(x[:, v]))
        x, err = y, e
    return x, err
