"""Plain 64-bit restatement of the training-step operators (numpy), sharing no code with the library:
8-bit matrices with a scale per 128 values, their products, the gradient norm, the AdamW step and the random
rounding of its 8-bit states.  Arithmetic and formats as include/cerar.h states them."""
import numpy as np

BLOCK, STATE_BLOCK = 128, 256
M32 = np.uint64(0xFFFFFFFF)


def e4m3_values():
    """The 256 values of the 8-bit format: sign, 4 exponent bits (bias 7), 3 mantissa bits, 0x7F and 0xFF are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = np.nan if c & 0x7F == 0x7F else (-mag if c & 0x80 else mag)
    return v


def spacing(y):
    """Distance of neighbouring codes at |y| (3 mantissa bits, 2^-9 below the smallest normal number)."""
    y = np.abs(np.asarray(y, dtype=np.float64))
    e = np.floor(np.log2(np.maximum(y, 2.0 ** -40)))
    return 2.0 ** np.maximum(e - 3, -9)


def scale_of(amax):
    """2^e, the smallest integer e in [-100, 100] with amax 2^-e <= 448; 1 for zero."""
    amax = np.asarray(amax, dtype=np.float64)
    _, e = np.frexp(amax / 448.0)                     # amax / 448 = f 2^e, f in [0.5, 1)
    e = np.where(amax / 448.0 == 2.0 ** (e - 1.0), e - 1, e)
    return np.where(amax > 0, 2.0 ** np.clip(e, -100, 100).astype(np.float64), 1.0)


def quantize(x, rows, cols):
    """(values of the codes, scales) of x with a scale per rows x cols values; NaN where x is not finite."""
    x = np.asarray(x, dtype=np.float64)
    r, c = x.shape
    nr, nc = -(-r // rows), -(-c // cols)
    q, s = np.empty_like(x), np.empty((nr, nc))
    mag = np.where(np.isfinite(x), np.abs(x), 0.0)
    for i in range(nr):
        band = np.maximum.reduceat(mag[i * rows:(i + 1) * rows].max(0), np.arange(0, c, cols))
        s[i] = scale_of(band)
        wide = np.repeat(s[i], cols)[:c]
        y = x[i * rows:(i + 1) * rows] / wide
        with np.errstate(invalid="ignore"):
            d = spacing(np.where(np.isfinite(y), y, 0.0))
            v = np.round(y / d) * d                   # numpy rounds halves to even
        q[i * rows:(i + 1) * rows] = np.where(np.isfinite(y), np.clip(v, -448, 448), np.nan)
    return q, s


def dequantize(q, s, rows, cols):
    return q * np.repeat(np.repeat(s, rows, 0), cols, 1)[:q.shape[0], :q.shape[1]]


def scramble(h):
    """Shifts and multipliers: C. Wellons, "Prospecting for Hash Functions", 2018."""
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x7FEB352D)) & M32
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0x846CA68B)) & M32
    return h ^ (h >> np.uint64(16))


def random_bits(first_block, n, seed, stream):
    """32 random bits for each of n elements of a tensor whose first state block has this number in the set."""
    nb = -(-n // STATE_BLOCK)
    b = np.arange(first_block, first_block + nb, dtype=np.uint64)
    with np.errstate(over="ignore"):
        key = (b & M32) * np.uint64(0x9E3779B1) + ((b >> np.uint64(32)) + np.uint64(1)) * np.uint64(0x7FEB352D)
        key += np.uint64(seed & 0xFFFFFFFF) * np.uint64(0x85157AF5) + np.uint64(seed >> 32) * np.uint64(0xC2B2AE35)
        key = scramble((key + np.uint64(stream) * np.uint64(0x632BE5AB)) & M32)
        lane = np.arange(STATE_BLOCK, dtype=np.uint64) * np.uint64(0x9E3779B9)
        return scramble((key[:, None] + lane[None, :]) & M32).reshape(-1)[:n]


def random_round(y, bits16):
    """y / spacing as a real number plus the random offset: the kept value is floor of it, times the spacing."""
    return np.abs(y) / spacing(y) + (np.asarray(bits16, np.float64) + 0.5) / 65536


def adamw(p, g, m, v, *, lr, beta1, beta2, eps, decay, step, coef=1.0):
    g = coef * np.asarray(g, np.float64)
    m = beta1 * np.asarray(m, np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, np.float64) + (1 - beta2) * g * g
    up = lr / (1 - beta1 ** step) * m / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    p = np.asarray(p, np.float64)
    return p - lr * decay * p - up, m, v, up


def grad_norm(grads, max_norm):
    n = float(np.sqrt(sum(float(np.sum(np.asarray(g, np.float64) ** 2)) for g in grads)))
    finite = np.isfinite(n)
    return n, (min(1.0, max_norm / (n + 1e-6)) if max_norm > 0 else 1.0) if finite else 0.0, float(finite)
