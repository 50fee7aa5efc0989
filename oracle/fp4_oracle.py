"""Plain float64 NumPy statement of microscaled 4-bit floating point (E2M1 codes; E8M0 scales of 32 channels, or E4M3 scales of
16 and a float32 scale a row) and of the norms around a block.  Only the tests use it."""

import numpy as np

MX, NV = 0, 1
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(c % 8) / 512.0 if c < 8 else (1 + c % 8 / 8.0) * 2.0 ** (c // 8 - 7) for c in range(127)])  # 0 .. 448
BLOCK = {MX: 32, NV: 16}


def nearest(x, numbers):
    """Index of the nearest of the ascending `numbers`, a tie to the even index, beyond the last to it; x >= 0."""
    hi = np.clip(np.searchsorted(numbers, x), 1, len(numbers) - 1)
    up, down = numbers[hi] - x, x - numbers[hi - 1]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)


def hadamard32(x, b):
    """Blocks of b channels times H / sqrt(b) as the kernels compute it: float32 butterflies of distance b/2 .. 1, one product."""
    x = np.asarray(x, np.float32)
    if b == 1:
        return x
    shape, h = x.shape, b // 2
    while h >= 1:
        y = x.reshape(-1, 2, h)
        x = np.stack((y[:, 0] + y[:, 1], y[:, 0] - y[:, 1]), 1)
        h //= 2
    return x.reshape(shape) * np.float32(1.0 / np.sqrt(b))


def quantize(z, fmt, step=None):
    """Finite float32 rows z to (codes uint8 [m, k], scale bytes uint8 [m, blocks], Delta float32 [m]); the quotients of float32
    numbers are taken in float64, where one that is no tie stays on its side of every tie."""
    z = np.asarray(z, np.float32)
    m, k = z.shape
    zb = z.reshape(m, -1, BLOCK[fmt]).astype(np.float64)
    top = np.abs(zb).max(-1)
    if fmt == MX:
        e = np.maximum(np.frexp(top)[1] - 3, -127)
        scale, unit, delta = np.where(top > 0, e + 127, 0), np.ldexp(1.0, e), np.ones(m, np.float32)
        unit = np.where(top > 0, unit, 0.0)
    else:
        delta = np.abs(z).max(-1) / np.float32(2688) if step is None else np.full(m, step, np.float32)
        d = delta.astype(np.float64)[:, None]
        scale = nearest(np.divide(top, 6 * d, out=np.zeros_like(top), where=d > 0), E4M3)
        unit = (E4M3[scale].astype(np.float32) * delta[:, None]).astype(np.float64)
    q = np.divide(np.abs(zb), unit[..., None], out=np.zeros_like(zb), where=unit[..., None] > 0)
    codes = nearest(q, E2M1) + 8 * np.signbit(zb)
    return codes.reshape(m, k).astype(np.uint8), scale.astype(np.uint8), delta


def scale_values(scale, fmt):
    s = scale.astype(np.int64)
    if fmt == MX:
        return np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return np.append(E4M3, np.nan)[np.minimum(s & 127, 127)]


def values(codes, scale, fmt):
    """codes * block scales, float64 (exact)."""
    c = codes.astype(np.int64)
    v = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    return v * np.repeat(scale_values(scale, fmt), BLOCK[fmt], 1)


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack(q):
    return np.stack((q & 15, q >> 4), -1).reshape(q.shape[0], -1)


def to_tiles(scale, fill=0):
    """[m, blocks] to tiles of 128 rows x 4 blocks; bytes of no row are `fill`."""
    m, n = scale.shape
    padded = np.full((-(-m // 128) * 128, n), fill, np.uint8)
    padded[:m] = scale
    return padded.reshape(-1, 4, 32, n // 4, 4).transpose(0, 3, 2, 1, 4).reshape(-1).copy()


def from_tiles(tiles, m, n):
    return tiles.reshape(-1, n // 4, 32, 4, 4).transpose(0, 3, 2, 1, 4).reshape(-1, n)[:m]


def gelu(x):
    return 0.5 * x * (1 + np.tanh(np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)))


def norm(x, layer, eps):
    x = np.asarray(x, np.float64)
    d = x - x.mean(-1, keepdims=True) if layer else x
    return d / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
