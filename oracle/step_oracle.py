"""An AdamW step in fp64 from its definition, and states in 8 bits as their rounding is defined, number for number.  NumPy only."""
import numpy as np

BLOCK = 256
M_FORMAT, V_FORMAT = (3, 7, 8), (2, 15, 15)        # mantissa bits, bias, and the exponent of the largest value, 1.75 2^top


def adamw(p, g, m, v, step, rate, betas, eps, decay, norm=None, max_norm=np.inf):
    """(p', m', v') in fp64."""
    if norm is not None and norm > max_norm:
        g = g * (max_norm / norm)
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    m_hat, v_hat = m / (1 - betas[0] ** step), v / (1 - betas[1] ** step)
    return p * (1 - rate * decay) - rate * m_hat / (np.sqrt(v_hat) + eps), m, v


def moments32(g, m, v, betas, clip=1.0):
    """m' and v' in fp32, every product and sum rounded by itself."""
    f = np.float32
    g = (g * f(clip)).astype(f)
    return m * f(betas[0]) + g * f(1 - betas[0]), v * f(betas[1]) + (g * g) * f(1 - betas[1])


def scramble(x):
    """PCG's RXS-M-XS permutation of 32-bit words as a hash."""
    x = np.asarray(x, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    s = (x * np.uint64(747796405) + np.uint64(2891336453)) & low
    w = (((s >> ((s >> np.uint64(28)) + np.uint64(4))) ^ s) * np.uint64(277803737)) & low
    return (w >> np.uint64(22)) ^ w


def words(at, seed, step, tensor):
    """A random word for every element number of `at`."""
    low = 0xFFFFFFFF
    key = scramble((int(scramble((seed + int(scramble(step & low))) & low)) + tensor) & low)
    at = np.asarray(at, dtype=np.uint64)
    high = at >> np.uint64(32)
    key = np.where(high != 0, key ^ scramble(high), key)
    return scramble((at & np.uint64(low)) ^ key)


def scales(x, top):
    """The smallest power of two, at least 2^-126, for which a block's largest value is at most 1.75 2^top (fp32, one a block of BLOCK)."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    x = np.where(np.isfinite(x), x, 0.0)
    most = np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK).max(1)
    with np.errstate(divide="ignore"):
        e = np.ceil(np.log2(most / (1.75 * 2.0 ** top)))
    return 2.0 ** np.maximum(e, -126)


def codes(x, r, mantissa, bias):
    """x >= 0 (already divided by its scale) as 8-bit codes, rounded up with the probability of its distance from the code below, by 16 random bits."""
    x = np.asarray(x, dtype=np.float64)
    e = np.maximum(np.floor(np.log2(np.maximum(x, 2.0 ** -200))), 1 - bias)
    steps = x / 2.0 ** (e - mantissa)                               # in steps of the code, [2^mantissa, 2^(mantissa + 1)) of a normal one
    whole = np.floor(steps + r / 65536.0)
    return np.where(x > 0, whole + (e + bias - 1) * 2 ** mantissa, 0).astype(np.int64)


def value(code, mantissa, bias):
    code = np.asarray(code, dtype=np.int64)
    e, f = code >> mantissa, code & (2 ** mantissa - 1)
    return np.where(e == 0, f * 2.0 ** (1 - bias - mantissa), (2 ** mantissa + f) * 2.0 ** (e - bias - mantissa))


def states8(m, v, w):
    """Codes and scales of m' and v' (fp32 values) with the random words w: (m codes, v codes, m scales, v scales)."""
    sm, sv = scales(m, M_FORMAT[2]), scales(v, V_FORMAT[2])
    x, y = np.asarray(m, dtype=np.float64) / np.repeat(sm, BLOCK)[:len(m)], np.asarray(v, dtype=np.float64) / np.repeat(sv, BLOCK)[:len(v)]
    a = codes(np.where(np.isfinite(x), np.abs(x), 0), (w >> np.uint64(16)).astype(np.float64), *M_FORMAT[:2])
    b = codes(np.where(np.isfinite(y), y, 0), (w & np.uint64(0xFFFF)).astype(np.float64), *V_FORMAT[:2])
    a = np.where(np.isfinite(x), np.minimum(a, 0x7E), 0x7F) + 128 * np.signbit(m)
    b = np.where(np.isfinite(y), np.maximum(np.minimum(b, 0x7B), y > 0), 0x7F)
    return a, b, sm, sv
