"""Inputs for which every sum of a microscaled 4-bit product is exact in fp32, so
that results can be required to be equal however long the inner axis is: a
tolerance that covers an fp32 sum of many terms would let a lost block of 32
through.  Test infrastructure only (numpy, no library code).

Values are +-{1, 2, 3, 4, 6}, doubled or not for each 32 x 32 tile of the matrix.
4-bit codes hold them along either axis and from any first row on: the block's
scale is 1 or 2 (or less, where all of it is small), and 1 / 2, 3 / 2 and 12 / 2 are
elements as well as 1, 3 and 6.  Products are whole numbers up to 144, so sums of
up to 2^24 / 144 of them are exact in any order.
"""
import numpy as np

MOST_TERMS = (1 << 24) // 144

# rows, columns, inner axis of products whose inner axis is long; all but the second are split
LONG = [(16, 16, 20500), (17, 33, 8200), (70, 130, 11000), (128, 1024, 12288), (64, 640, 30000)]


def held(rng, *shape):
    """[..., rows, cols] in float32"""
    *lead, rows, cols = shape
    v = rng.choice(np.array([1, 2, 3, 4, 6], np.float32), shape) * rng.choice(np.array([-1, 1], np.float32), shape)
    double = rng.integers(1, 3, (*lead, -(-rows // 32), -(-cols // 32))).astype(np.float32)
    return v * double.repeat(32, -2).repeat(32, -1)[..., :rows, :cols]


def operands(M, N, K):
    """The pair of a case of LONG."""
    rng = np.random.default_rng(M + 7 * N + 13 * K)
    return held(rng, M, K), held(rng, N, K)


def equal(got, a, b):
    """got = a b^T (tensors), the sums in 64 bits, rounded once to got's type."""
    import torch
    assert a.shape[1] <= MOST_TERMS
    want = a.double() @ b.double().t().contiguous()
    assert torch.equal(got, want.float().to(got.dtype))
