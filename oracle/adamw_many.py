"""AdamW over separate tensors with moments in 32 or 8 bits (test infrastructure), in fp64 with numpy.

8 bits: 256 consecutive values share top_m = max |m| and top_v = max v (kept in fp32);
m = sign(c) (c / 127)^2 top_m and v = (c / 255)^4 top_v.  Of the two codes around a value the upper one is taken if the
number of its place, in (0, 1), is below the share of the way from the lower value to the upper; a positive v keeps code 1
at least.  The numbers are two halves of a mixed 32-bit counter of seed, step and place."""
import numpy as np

BLOCK = 256


def numbers(places, t, seed):
    """(for m, for v)."""
    low = np.uint64(0xFFFFFFFF)
    p = np.asarray(places, np.uint64)
    x = ((p & low) * np.uint64(0x9E3779B1) + (p >> np.uint64(32)) * np.uint64(0x85EBCA77)
         + np.uint64(t * 0xC2B2AE3D % 2 ** 32 + seed)) & low
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x46A2CA6B)) & low
    x ^= x >> np.uint64(16)
    return ((x & np.uint64(0xFFFF)).astype(np.float64) + 0.5) / 65536, ((x >> np.uint64(16)).astype(np.float64) + 0.5) / 65536


def _blocks(x):
    pad = -len(x) % BLOCK
    return np.concatenate([x, np.zeros(pad)]).reshape(-1, BLOCK)


def encode(x, most, power, least, u, top=None):
    """(codes with the sign of x, tops in fp32) of the values x; top: scales to use instead of the blocks' own."""
    n = len(x)
    b = _blocks(np.asarray(x, np.float64))
    top = np.abs(b).max(axis=1).astype(np.float32) if top is None else top
    unit = np.repeat(top.astype(np.float64), BLOCK)[:n] / float(most) ** power
    y = np.abs(np.asarray(x, np.float64))
    ladder = np.arange(most + 2, dtype=np.float64) ** power
    with np.errstate(all="ignore"):
        share = np.where(unit > 0, y / unit, 0.0)
    c = np.clip(np.searchsorted(ladder, share, side="right") - 1, 0, most)
    way = (share - ladder[c]) / (ladder[c + 1] - ladder[c])
    c = np.where((c < most) & (u < way), c + 1, c)
    c = np.where((y > 0) & (unit > 0), np.maximum(c, least), np.where(unit > 0, c, 0))
    return (np.sign(x) * c).astype(np.int64), top


def decode(c, top, most, power):
    c = np.asarray(c, np.float64)
    return np.sign(c) * (np.abs(c) / most) ** power * np.repeat(np.asarray(top, np.float64), BLOCK)[:len(c)]


def coefficient(sq, clip):
    return min(1.0, clip / (np.sqrt(sq) + 1e-6))


def step(theta, grad, m, v, t, *, lr, beta1, beta2, eps, decay, coef):
    """theta, m, v after step number t, all fp64; decay is this tensor's."""
    g = np.asarray(grad, np.float64) * coef
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    theta = theta - lr * (decay * theta + m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps))
    return theta, m, v
