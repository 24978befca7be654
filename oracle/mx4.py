"""Oracle of the microscaled 4-bit operators: numpy in fp64, written from the definitions in include/defl.h. Values are handled
as numbers, not codes; `encode` and `tiles` give the bytes they are held in."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"mxfp4": 32, "nvfp4": 16}


def _e4m3_grid():
    """All e4m3 values that are not negative, by their byte (the last one, NaN, left out)."""
    out = []
    for byte in range(127):
        e, f = byte >> 3, byte & 7
        out.append(2.0 ** (e - 7) * (1 + f / 8) if e else 2.0 ** -6 * f / 8)
    return np.array(out)


E4M3 = _e4m3_grid()


def nearest_even(x, grid):
    """Index of the grid value nearest to each x >= 0; a tie goes to the even index, what is above the grid to its end."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    up, down = grid[hi] - x, x - grid[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def whole_scale(X, fmt):
    """The matrix's own scale: the smallest power of two (from 2^-100 on) with |X| <= 6 * 448 * 2^w, from the values that are finite."""
    if fmt == "mxfp4":
        return 1.0
    a = np.abs(X[np.isfinite(X)])
    top = a.max() if a.size else 0.0
    if top == 0.0:
        return 1.0
    w = -100
    while top > 2688.0 * 2.0 ** w:
        w += 1
    return 2.0 ** w


def quantize(X, fmt):
    """(signed grid index, scale byte per block, matrix scale) of one matrix, blocks along the last dimension."""
    X = np.asarray(X, dtype=np.float64)
    rows, cols = X.shape
    blk = BLOCK[fmt]
    width = (cols + 31) // 32 * 32
    P = np.zeros((rows, width))
    P[:, :cols] = X
    P = P.reshape(rows, width // blk, blk)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(P).all(axis=2)
    Q = np.where(bad[:, :, None], 0.0, P)
    big = np.abs(Q).max(axis=2)
    whole = whole_scale(X, fmt)
    if fmt == "mxfp4":
        e = np.full(big.shape, -127)
        some = big > 0
        frac, ex = np.frexp(np.where(some, big, 1.0))            # big = frac 2^ex, frac in [1/2, 1): 6 * 2^e = .75 * 2^(e + 3)
        e = np.where(some, np.maximum(np.where(frac <= 0.75, ex - 3, ex - 2), -127), e)
        byte = (e + 127).astype(np.uint8)
        scale = np.ldexp(1.0, e)
        byte = np.where(bad, 255, byte).astype(np.uint8)
    else:
        quotient = (np.float32(1.0) * (big / whole).astype(np.float32) / np.float32(6.0)).astype(np.float64)   # a fp32 quotient by definition
        byte = nearest_even(quotient, E4M3).astype(np.uint8)
        scale = E4M3[byte] * whole
        byte = np.where(bad, 0x7F, byte).astype(np.uint8)
    ratio = np.where(scale[:, :, None] > 0, Q / np.where(scale > 0, scale, 1.0)[:, :, None], 0.0)
    index = nearest_even(np.abs(ratio), GRID) * np.where(Q < 0, -1, 1)
    return index.reshape(rows, width), byte, whole


def decode_scale(byte, fmt, whole):
    byte = np.asarray(byte, dtype=np.int64)
    if fmt == "mxfp4":
        return np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))
    return np.where(byte == 0x7F, np.nan, E4M3[np.minimum(byte, 126)] * whole)


def values(index, byte, whole, fmt, cols):
    """What the codes stand for, in fp64."""
    rows, width = index.shape
    v = np.sign(index) * GRID[np.abs(index)]
    s = decode_scale(byte, fmt, whole)
    return (v.reshape(rows, width // BLOCK[fmt], BLOCK[fmt]) * s[:, :, None]).reshape(rows, width)[:, :cols]


def round_trip(X, fmt):
    return values(*quantize(X, fmt), fmt, X.shape[1])


def pack(nibbles):
    """Two codes a byte, the even column in the low half."""
    return (nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)).astype(np.uint8)


def tiles(byte):
    """Scale bytes [rows, blocks] in tiles of 128 rows x 4 blocks, 512 bytes each."""
    rows, nb = byte.shape
    rt, kt = -(-rows // 128), -(-nb // 4)
    out = np.zeros((rt, kt, 512), dtype=np.uint8)
    for r in range(rows):
        for c in range(nb):
            out[r // 128, c // 4, (r % 32) * 16 + (r % 128) // 32 * 4 + c % 4] = byte[r, c]
    return out
