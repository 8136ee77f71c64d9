"""fp32 factors in three bf16 parts: numbers on which every product of parts counts, and how far products may be off."""
import numpy as np

# |error| of one product of two fp32 factors taken in bf16 parts, over the product, in u: six products, each added
# in fp32 (at most a whole step, 2 u), and the three that are left out (2^-8 2^-17 twice, 2^-17 2^-17: under 2 u).
PARTS = 6 * 2 + 2


def three_parts():
    """Two fp32 numbers whose second and third bf16 parts are as large as they get, of one sign."""
    x = np.float32(1 + (2.0 ** -8 - 2.0 ** -16) + (2.0 ** -17 - 2.0 ** -23))
    y = np.float32(1 + (2.0 ** -8 - 2.0 ** -15) + (2.0 ** -17 - 2.0 ** -22))
    return x, y


def bf16(v):
    """To the nearest bf16, ties to even."""
    b = np.asarray(v, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7fff + (b >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def parts_of(v):
    v, out = np.float32(v), []
    for _ in range(3):
        p = np.float32(bf16(v))
        out.append(float(p))
        v = np.float32(v - p)
    return out, float(v)
