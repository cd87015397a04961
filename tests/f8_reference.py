"""Plain implementation in 64 bits of the 8-bit floating-point format with a scale
for each block of 128, from the definitions in include/shiftquant.h.  Test
infrastructure only (numpy, no library code)."""
import numpy as np

# the values of the codes 0 .. 126 (127 is no number)
E4M3 = np.array([(k & 7) * 2.0 ** -9 if k < 8 else (8 + (k & 7)) * 2.0 ** ((k >> 3) - 10) for k in range(127)])


def _scale_bytes(a):
    """Smallest s in 0 .. 254 with a / 2^(s - 127) <= 464; 255 where a is not finite."""
    s = np.full(a.shape, 254)
    for cand in range(253, -1, -1):
        s = np.where(np.where(np.isfinite(a), a, 0.0) / 2.0 ** (cand - 127) <= 464.0, cand, s)
    return np.where(np.isfinite(a), s, 255)


def scale_bytes(x, square=False):
    """The scale byte of every element of x [rows, cols]."""
    rows, cols = x.shape
    b = np.zeros((-(-rows // 128) * 128, -(-cols // 128) * 128))
    b[:rows, :cols] = np.abs(np.where(np.isnan(x), np.inf, x))
    m = b.reshape(b.shape[0], -1, 128).max(2)
    if square:
        m = np.repeat(m.reshape(-1, 128, m.shape[1]).max(1), 128, 0)
    return np.repeat(_scale_bytes(m), 128, 1)[:rows, :cols]


def f8_codes(x, square=False):
    """(codes, scale bytes) of every element of x [rows, cols]"""
    x = np.asarray(x, np.float64)
    s = scale_bytes(x, square)
    v = np.where(s == 255, 0.0, x) / 2.0 ** (np.where(s == 255, 127, s) - 127.0)
    a = np.abs(v)
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)              # E4M3[hi - 1] <= a <= E4M3[hi], or past the last
    lo = hi - 1
    down, up = a - E4M3[lo], E4M3[hi] - a
    k = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))     # a tie goes to the even code
    return np.where(s == 255, 0, k | (np.signbit(v) << 7)).astype(np.uint8), s.astype(np.uint8)


def f8_values(x, square=False):
    """The values that f8_codes stand for."""
    k, s = f8_codes(x, square)
    v = np.where(k & 128, -1.0, 1.0) * E4M3[k & 127] * 2.0 ** (s.astype(np.float64) - 127)
    return np.where(s == 255, np.nan, v)


def f8_places(rows, cols):
    """Byte and scale byte of every element [rows, cols] of a matrix (the documented layout)."""
    r, k = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    unit = (r // 16) * -(-cols // 512) + k // 512
    return (unit * 8192 + (k // 128) % 4 * 2048 + (k // 16) % 8 * 256 + (r % 16) * 16 + k % 16,
            unit * 64 + (r % 16) * 4 + (k // 128) % 4)


def held(rng, *shape):
    """Whole numbers that the codes hold along either axis, whatever block they are in: +-{1, 2, 3, 4, 6, 8, 12, 15},
    products at most 225, so that sums of 2^24 / 225 of them are exact in fp32 in any order.  (Scales are at most 1 / 16
    of the largest element's power of two, so that even 1 is a normal element.)"""
    return rng.choice([1, 2, 3, 4, 6, 8, 12, 15], shape) * rng.choice([-1, 1], shape)
