"""Oracle of the AdamW step and of the gradient norm: numpy in fp64, written from the formulas in include/defl.h.

The moments in 8 bits are handled as numbers (e4m3 values, not codes), so nothing here shares a table or a bit trick with
the kernels; the random bits are an input and come from `random_bits`, the documented generator in 64-bit integers.
"""
import numpy as np

BLOCK = 256
TOP = 448.0                 # largest e4m3 magnitude
LEAST = 2.0 ** -9           # smallest one that is not zero
FLUSH = 2.0 ** -100         # blocks whose largest magnitude is below count as zero


def _h(x):
    x = np.asarray(x, dtype=np.uint64) + np.uint64(0x9E3779B97F4A7C15)
    x = (x ^ (x >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    x = (x ^ (x >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return x ^ (x >> np.uint64(31))


def random_bits(seed, t, index, n):
    """(bits for m, bits for the root and a bf16 weight): 16 each for the n elements of list entry `index` at step t."""
    with np.errstate(over="ignore"):
        key = _h(_h(_h(np.uint64(seed)) ^ np.uint64(t)) ^ np.uint64(index))
        word = _h(key ^ np.arange((n + 1) // 2, dtype=np.uint64))
    half = np.stack([word & np.uint64(0xFFFFFFFF), word >> np.uint64(32)], axis=1).reshape(-1)[:n]
    return (half & np.uint64(0xFFFF)).astype(np.int64), (half >> np.uint64(16)).astype(np.int64)


def e4m3_spacing(y):
    """Distance of neighbouring e4m3 values at y >= 0."""
    _, e = np.frexp(np.maximum(y, 2.0 ** -6))
    return np.ldexp(1.0, e - 4)


def e4m3_stochastic(y, bits):
    d = e4m3_spacing(y)
    return np.minimum(np.floor(y / d + bits / 65536.0) * d, TOP)


def e4m3_nearest(y):
    d = e4m3_spacing(y)
    return np.minimum(np.rint(y / d) * d, TOP)          # rint: ties to even, and an even multiple of d is an even mantissa


def bf16_stochastic(x, bits):
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** -126))
    d = np.ldexp(1.0, e - 8)
    return np.sign(x) * np.floor(np.abs(x) / d + bits / 65536.0) * d


def scaled_blocks(x):
    """(y = |x| * 448 / largest of the block, scale per block) of a vector."""
    n = x.size
    nb = (n + BLOCK - 1) // BLOCK
    a = np.zeros(nb * BLOCK)
    a[:n] = np.abs(x)
    big = a.reshape(nb, BLOCK).max(axis=1) if nb else np.zeros(0)
    inv = np.where(big > FLUSH, TOP / np.where(big > FLUSH, big, 1.0), 0.0)
    return (a.reshape(nb, BLOCK) * inv[:, None]).reshape(-1)[:n], np.where(big > FLUSH, big / TOP, 0.0)


def store8(x, bits, keep_nonzero):
    """(e4m3 values with sign, scales); bits None: to nearest."""
    y, scale = scaled_blocks(x)
    z = e4m3_nearest(y) if bits is None else e4m3_stochastic(y, bits)
    if keep_nonzero:
        z = np.where(y > 0, np.maximum(z, LEAST), z)
    return np.sign(x) * z, scale


def load8(q, scale):
    return q * np.repeat(scale, BLOCK)[:q.size]


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, c=1.0):
    """(p, m, v) after step t >= 1."""
    g = c * g
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    mhat, vhat = m / (1.0 - beta1 ** t), v / (1.0 - beta2 ** t)
    return (1.0 - lr * weight_decay) * p - lr * mhat / (np.sqrt(vhat) + eps), m, v


def grad_norm(grads, max_norm):
    """(norm, factor) of a list of arrays."""
    norm = float(np.sqrt(sum(float(np.sum(np.square(g, dtype=np.float64))) for g in grads)))
    if not np.isfinite(norm):
        return norm, 0.0
    return norm, min(1.0, max_norm / (norm + 1e-6)) if max_norm > 0 else 1.0
