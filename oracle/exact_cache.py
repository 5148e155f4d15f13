"""The 8-bit cache of exact keys and values, and attention over it, in fp64 from the definitions in include/kvm.h (numpy only)."""
import numpy as np

LEAST_EXP = -64


def _e4m3_table():
    """The non-negative finite values of e4m3 in the order of their codes: subnormals m/8 * 2^-6, then (1 + m/8) * 2^(e-7), up to 448."""
    sub = [m / 8.0 * 2.0 ** -6 for m in range(8)]
    nor = [(1 + m / 8.0) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(sub + nor[:-1])   # (the last code is NaN)


E4M3 = _e4m3_table()


def round_e4m3(x):
    """Nearest value of e4m3, ties to the even code; |x| <= 448."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    hi = np.searchsorted(E4M3, a).clip(0, len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(E4M3[code], x)


def least_exp(amax):
    """Least e >= -64 with amax <= 448 * 2^e."""
    if amax == 0:
        return LEAST_EXP
    e = int(np.floor(np.log2(amax / 448.0))) - 1
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return max(e, LEAST_EXP)


class Block:
    """One page of one head, keys or values: code values [P, d] and the exponent of the scale (None: NaN)."""

    def __init__(self, P, d):
        self.code, self.exp, self.rows = np.zeros((P, d)), LEAST_EXP, 0

    def add(self, x):
        x = np.asarray(x, np.float64)
        if not np.isfinite(x).all() or self.exp is None:
            self.exp = None
        else:
            e = max(self.exp, least_exp(np.abs(x).max()))
            self.code[:self.rows] = round_e4m3(self.code[:self.rows] * 2.0 ** (self.exp - e))
            self.code[self.rows:self.rows + len(x)] = round_e4m3(x * 2.0 ** -e)
            self.exp = e
        self.rows += len(x)

    def values(self):
        return self.code[:self.rows] * (np.nan if self.exp is None else 2.0 ** self.exp)


class Rows:
    """The rows of one sequence and head (keys or values), appended call by call."""

    def __init__(self, P, d):
        self.P, self.d, self.blocks = P, d, []

    def add(self, x):
        at = 0
        while at < len(x):
            if not self.blocks or self.blocks[-1].rows == self.P:
                self.blocks.append(Block(self.P, self.d))
            n = min(len(x) - at, self.P - self.blocks[-1].rows)
            self.blocks[-1].add(x[at:at + n])
            at += n

    def values(self):
        return np.concatenate([b.values() for b in self.blocks]) if self.blocks else np.zeros((0, self.d))


def attend(q, k, v, pos, scale, window=0, sinks=0):
    """Rows q [n, d] at positions pos [n] over keys and values [L, d]: (out [n, d], bound on a kernel's error [n, d]).

    The bound counts, besides half a step of bf16 (2^-8 of the result) for the output:
    - the logits: products of bf16 and e4m3 are exact in fp32, a sum of 2 d of them (q in two parts) loses at most 2 d * 2^-23 of the sum of
      magnitudes, twice that for scaling and exponent arithmetic; what q's two parts of 8 bits leave of channels far below its largest
      is at most 2^-18 of that; a logit error of x changes a weight by a factor of e^x;
    - the weights: two parts of e4m3 keep 2^-8 of a weight, and 2^-18 of the largest one of its tile of 128 keys where they
      are subnormal (one part of fp16 keeps more): together at most 2^-8 of the sum of |p v| and 2^-11 of the largest |v|;
    - fp32 sums over the keys: 2^-20 of the sum of |p v|."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    j = np.arange(len(k))[None]
    p = np.asarray(pos)[:, None]
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    z = np.where(see, q @ k.T * scale, -np.inf)
    w = np.exp(z - z.max(1, keepdims=True))
    w = np.where(see, w / w.sum(1, keepdims=True), 0.0)
    vis = see.any(0)
    vz = np.where(vis[:, None], v, 0.0)
    out = w @ vz
    mag = scale * (np.abs(q) @ np.abs(k).T) * (4 * q.shape[1] * 2.0 ** -23) + scale * 2.0 ** -18 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1)[None]
    dz = np.where(see, mag, 0.0).max(1, keepdims=True)
    bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2.0 ** -20 + 2 * np.expm1(dz)) * (w @ np.abs(vz)) + 2.0 ** -11 * np.abs(vz).max()
    return out, bound
