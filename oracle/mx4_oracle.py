"""Oracle of the microscaled 4-bit operators: plain numpy in 64 bits, written from the format's definition.

A block of 32 values x has the scale 2^e, e = floor(log2 max|x|) - 2 held to [-127, 125]; its codes are the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| 2^-e (ties to the even code, larger values to the last) with the sign of x in bit 3.
A block with a NaN or an infinity has the scale byte 255 and zero codes and decodes to NaN.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode_blocks(x):
    """x [..., 32] (finite or not) -> (codes [..., 32] uint8, scale bytes [...] uint8)."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.clip(np.frexp(safe)[1] - 1 - 2, -127, 125)         # frexp: top = f 2^n, 0.5 <= f < 1
    e = np.where(top == 0, -127, e)
    t = np.ldexp(np.where(bad[..., None], 0.0, np.abs(x)), -e[..., None])
    dist = np.abs(t[..., None] - GRID)
    near = dist.min(-1, keepdims=True)
    tied = dist == near                                       # one code, or two neighbours
    pick = np.where(tied, np.arange(8), -1)
    hi = pick.max(-1)
    lo = np.where(tied, np.arange(8), 8).min(-1)
    code = np.where((hi != lo) & (hi % 2 == 1), lo, hi).astype(np.uint8)
    code |= np.where(np.signbit(x), 8, 0).astype(np.uint8)
    code[bad] = 0
    return code, np.where(bad, 255, e + 127).astype(np.uint8)


def decode_blocks(code, byte):
    """Values [..., 32] of codes and scale bytes."""
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))
    return v * scale[..., None]


def to_blocks(x):
    """[rows, cols] -> [rows, blocks, 32], zeros behind the last column."""
    x = np.asarray(x)
    rows, cols = x.shape
    nb = -(-cols // 32)
    out = np.zeros((rows, nb * 32), np.float64)
    out[:, :cols] = x
    return out.reshape(rows, nb, 32)


def pack(code):
    """[..., 32] codes -> [..., 16] bytes, element 2i in the low half of byte i."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def unpack(data):
    out = np.empty(data.shape[:-1] + (data.shape[-1] * 2,), np.uint8)
    out[..., 0::2], out[..., 1::2] = data & 15, data >> 4
    return out


def tile_scales(byte):
    """[rows, blocks] scale bytes -> the tiled layout, element by element."""
    rows, nb = byte.shape
    kt = -(-nb // 4)
    out = np.zeros(-(-rows // 128) * kt * 512, np.uint8)
    for r in range(rows):
        for j in range(nb):
            out[(r // 128 * kt + j // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4] = byte[r, j]
    return out


def quantize(x):
    """(codes bytes, tiled scales, values [rows, cols]) of a matrix along its rows."""
    rows, cols = np.asarray(x).shape
    code, byte = encode_blocks(to_blocks(x))
    return pack(code).reshape(-1), tile_scales(byte), decode_blocks(code, byte).reshape(rows, -1)[:, :cols]


def compress(grad, residual):
    """(codes, scales, values, residual) of a flat gradient; acc is one fp32 addition."""
    acc = (np.asarray(grad, np.float32) + np.asarray(residual, np.float32)).astype(np.float32)
    d = acc.size
    blocks = np.zeros(-(-d // 32) * 32, np.float64)
    blocks[:d] = acc
    code, byte = encode_blocks(blocks.reshape(-1, 32))
    value = decode_blocks(code, byte).reshape(-1)[:d]
    return pack(code).reshape(-1), byte, value, (acc.astype(np.float64) - value).astype(np.float32)


def mean(codes_all, scales_all, n_workers, d):
    """Dense mean in 64 bits."""
    nb = -(-d // 32)
    code = unpack(codes_all.reshape(n_workers, nb, 16))
    return decode_blocks(code, scales_all.reshape(n_workers, nb)).reshape(n_workers, -1)[:, :d].sum(0) / n_workers
