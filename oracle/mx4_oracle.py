"""Plain 64-bit form of the microscaled 4-bit format (numpy): the definition that the GPU kernels are compared with.

A block of 32 values shares 2^e, e = clamp(floor(log2 max|x|) - 2, -127, 127); a code is the E2M1 number nearest to
x / 2^e, ties to the even code, magnitudes above 6 to 6; a block that holds a NaN or an infinity stands for NaN."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """x [rows, k] of any floating type -> (codes uint8 [rows, k], one code per byte; scale bytes uint8 [rows, k/32])."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    b = x.reshape(rows, k // 32, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    top = np.abs(b).max(axis=2)
    _, ex = np.frexp(top)                                   # top = f * 2^ex, 1/2 <= f < 1: floor(log2 top) = ex - 1
    e = np.where(top > 0, np.clip(ex - 3, -127, 127), -127)
    y = np.abs(b) / np.exp2(e.astype(np.float64))[:, :, None]
    # nearest of eight magnitudes; of two that are as near, the even code
    dist = np.abs(y[..., None] - GRID)
    near = dist.min(axis=-1, keepdims=True)
    cand = dist == near
    even = cand & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), cand.argmax(axis=-1)).astype(np.uint8)
    code |= (np.signbit(b).astype(np.uint8) << 3)
    code = np.where(bad[:, :, None], 0, code).astype(np.uint8).reshape(rows, k)
    return code, np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    """The numbers that codes and scale bytes stand for, in 64 bits."""
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return v * np.repeat(s, 32, axis=1)


def pack(code):
    """Two codes to a byte, the even column low."""
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    out = np.empty((packed.shape[0], 2 * packed.shape[1]), dtype=np.uint8)
    out[:, 0::2], out[:, 1::2] = packed & 15, packed >> 4
    return out


def panels(scale):
    """Scale bytes [rows, k/32] in the stored order [ceil(k/256)][rows][8], zero beyond k."""
    rows, nb = scale.shape
    full = np.zeros((rows, -(-nb // 8) * 8), dtype=np.uint8)
    full[:, :nb] = scale
    return np.ascontiguousarray(full.reshape(rows, -1, 8).transpose(1, 0, 2))


def unpanels(stored, k):
    return np.ascontiguousarray(stored.transpose(1, 0, 2).reshape(stored.shape[1], -1)[:, :k // 32])
