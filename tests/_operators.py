"""Plain references in numpy, 64 bits, of microscaled 4-bit floating point and of the AdamW step, written from the formulas of
``include/zccl.h`` (no code of the package)."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
NIBBLES = np.concatenate([GRID, -GRID])


def quantize(x):
    """x [rows, cols] (any float type) -> values the codes stand for before scaling [rows, blocks, 32] and biased exponents [rows, blocks]."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    full = np.zeros((rows, blocks * 32))
    full[:, :cols] = x.astype(np.float64)
    b = full.reshape(rows, blocks, 32)
    bad = ~np.isfinite(b).all(-1)
    safe = np.where(bad[..., None], 0.0, b)
    top = np.abs(safe).max(-1)
    e = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))) - 2, -127)
    # log2 of a 64-bit number next to a power of two may round over it
    e = np.where((top > 0) & (np.ldexp(1.0, (e + 2).astype(int)) > top), e - 1, e)
    e = np.clip(e, -127, 127).astype(int)
    y = np.ldexp(safe, -e[..., None])
    a = np.abs(y)
    low = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    lo, hi = GRID[low], GRID[low + 1]
    middle = (lo + hi) / 2
    up = (a > middle) | ((a == middle) & (low % 2 == 1))     # ties to the even index: an even mantissa bit
    index = np.where(a >= 6, 7, low + up)
    s = np.where(bad, 255, e + 127)
    return np.where(bad[..., None], 0.0, np.copysign(GRID[index], y)), s


def scale_index(rows, blocks):
    """Where the scale of (row, block) stands."""
    r, b = np.meshgrid(np.arange(rows), np.arange(blocks), indexing="ij")
    return ((r // 128) * (-(-blocks // 4)) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def unpack(codes, scales, rows, cols):
    """Bytes -> (values before scaling [rows, blocks, 32], biased exponents [rows, blocks])."""
    blocks = -(-cols // 32)
    c = codes.reshape(rows, blocks, 16)
    v = np.stack([NIBBLES[c & 15], NIBBLES[c >> 4]], -1).reshape(rows, blocks, 32)
    return v, scales[scale_index(rows, blocks)].astype(int)


def pack(values, s):
    """The opposite of unpack (zeros keep their sign bit)."""
    rows, blocks, _ = values.shape
    n = np.searchsorted(GRID, np.abs(values)).astype(np.uint8) | (np.signbit(values).astype(np.uint8) << 3)
    codes = (n[..., 0::2] | (n[..., 1::2] << 4)).reshape(-1)
    scales = np.zeros(-(-rows // 128) * (-(-blocks // 4)) * 512, np.uint8)
    scales[scale_index(rows, blocks)] = s
    return codes, scales


def values(v, s, cols):
    out = np.where(s[..., None] == 255, np.nan, np.ldexp(v, np.where(s == 255, 0, s - 127)[..., None]))
    return out.reshape(out.shape[0], -1)[:, :cols]


# ---- AdamW

def random_bits(seed, step, place):
    """32 random bits for each element at `place` (uint64)."""
    with np.errstate(over="ignore"):
        key = np.uint64((seed + step * 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF)
        low, m = np.uint64(0xFFFFFFFF), np.uint64
        place = place.astype(np.uint64)
        h = ((place ^ key) & low) * m(0x7FEB352D) & low
        h = ((h ^ (h >> m(15))) ^ (key >> m(32)) ^ (place >> m(32))) * m(0x846CA68B) & low
        h = (h ^ (h >> m(13))) * m(0x6C8E9CF5) & low
        return h ^ (h >> m(16))


def encode8(x, random16, root):
    """x [n] -> (E4M3 values with sign [n], biased exponent per block), stochastic rounding."""
    n = x.size
    b = np.zeros(-(-n // 32) * 32)
    b[:n] = x
    b = b.reshape(-1, 32)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0.0, np.abs(b).max(-1))
    f, e = np.frexp(top)
    e = np.where(top > 0, np.maximum(e - 9 + (f > 0.875), -127), -127)
    y = np.ldexp(np.abs(b), -e[:, None]).reshape(-1)[:n]
    _, at = np.frexp(y)
    grid = np.ldexp(1.0, np.maximum(at - 4, -9))
    q = np.floor(y / grid + random16 / 65536.0) * grid
    if root:
        q = np.where(x > 0, np.maximum(q, 2.0 ** -9), q)
    return np.copysign(q, x), np.where(bad, 255, e + 127), grid * np.ldexp(1.0, np.repeat(e, 32)[:n])


def step_of(p, g, m, v, *, lr, betas, eps, weight_decay, step, norm=None, max_norm=1.0):
    """The updated (p, m, v) in 64 bits."""
    b1, b2 = betas
    if norm is not None:
        g = g * min(1.0, max_norm / (norm + 1e-6))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * weight_decay) - lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps), m, v
