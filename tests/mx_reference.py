"""Plain implementation in 64 bits of the microscaled 4-bit format, its products
and the activations with 8-bit copies, from the definitions in
include/shiftquant.h.  Test infrastructure only (numpy, no library code)."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _blocks(x):
    """Blocks of 32 of the last axis, zero padded, in float64."""
    x = np.asarray(x, np.float64)
    pad = -x.shape[-1] % 32
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (pad,))], -1)
    return x.reshape(x.shape[:-1] + (-1, 32))


def _scale_bytes(b, fits):
    """Smallest s in 0 .. 254 with fits(max |x| / 2^(s - 127)); 255 where a block is not finite."""
    bad = ~np.isfinite(b).all(-1)
    a = np.where(bad[..., None], 0.0, np.abs(b)).max(-1)
    s = np.full(a.shape, 254)
    for cand in range(253, -1, -1):
        s = np.where(fits(a / 2.0 ** (cand - 127)), cand, s)
    return np.where(bad, 255, s).astype(np.uint8)


def mx_codes(x):
    """(codes [..., blocks, 32] in 0 .. 15, scale bytes [..., blocks])"""
    b = _blocks(x)
    s = _scale_bytes(b, lambda r: r <= 7.0)
    v = np.where(s[..., None] == 255, 0.0, b) / 2.0 ** (np.where(s == 255, 127, s).astype(np.int64) - 127)[..., None]
    d = np.abs(np.abs(v)[..., None] - E2M1)             # distance to every element
    near = d == d.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    k = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))    # a tie goes to the even code
    return (k | (np.signbit(v) << 3)).astype(np.uint8), s


def mx_values(x):
    """The values [..., cols] that mx_codes stand for."""
    k, s = mx_codes(x)
    v = np.where(k & 8, -1.0, 1.0) * E2M1[k & 7] * 2.0 ** (s.astype(np.int64) - 127)[..., None]
    v = np.where(s[..., None] == 255, np.nan, np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v))
    return v.reshape(v.shape[:-2] + (-1,))[..., :np.shape(x)[-1]]


def mx_places(rows, cols):
    """Byte, nibble and scale byte of every element [rows, cols] of a matrix (the documented layout)."""
    r, k = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    units = -(-cols // 512)
    unit = (r // 16) * units + k // 512
    byte = unit * 4096 + (k // 128) % 4 * 1024 + (k // 32) % 4 * 256 + (r % 16) * 16 + (k % 32) // 2
    return byte, k % 2, unit * 256 + (k // 32) % 4 * 64 + (r % 16) * 4 + (k // 128) % 4


def mx_unpack(codes, scales, rows, cols):
    """(codes [rows, cols], scale bytes [rows, cols]) out of the buffers of a matrix."""
    byte, nib, sc = mx_places(rows, cols)
    return (codes[byte] >> (4 * nib)) & 15, scales[sc]


def segments(offsets):
    return list(zip(offsets[:-1], offsets[1:]))


def mx_product(a, b):
    """Sum over the last axis of both, and the sum of the magnitudes."""
    return a @ b.T, np.abs(a) @ np.abs(b).T


def copy8(x):
    """The values that the 8-bit copy of x [..., F] holds."""
    b = _blocks(x)
    s = _scale_bytes(b, lambda r: r < 127.5)
    step = 2.0 ** (np.where(s == 255, 127, s).astype(np.int64) - 127)[..., None]
    code = np.rint(np.where(s[..., None] == 255, 0.0, b) / step)
    v = np.where(s[..., None] == 255, np.nan, code * step)
    return v.reshape(v.shape[:-2] + (-1,))[..., :np.shape(x)[-1]], code, s


def act(kind, x):
    """act(x) in float64"""
    if kind == "silu":
        return x / (1.0 + np.exp(-x))
    return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def act_slope(kind, x):
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-x))
        return s * (1.0 + x * (1.0 - s))
    k = math.sqrt(2.0 / math.pi)
    t = np.tanh(k * (x + 0.044715 * x ** 3))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * x * x)
