"""Linear layers in 4 bits and the optimiser's step, in fp64 from their definitions.

A 4-bit matrix: e2m1 values and a scale for every 16 (e4m3) or 32 (a power of two, e8m0)
columns of a row, e4m3 scales times 2^exponent; see include/refadapt.h for the layout.
"""
import numpy as np

E4M3, E8M0 = 0, 1
BLOCK = {E4M3: 16, E8M0: 32}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _e4m3_table():
    """The 127 non-negative finite values, by code."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


E4M3_VALUES = _e4m3_table()


def nearest(x, grid):
    """Codes of the grid's values nearest to x >= 0, of two the even one, at most the last."""
    x = np.minimum(np.asarray(x, np.float64), grid[-1])
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    middle = 0.5 * (grid[lo] + grid[hi])
    up = (x > middle) | ((x == middle) & (hi % 2 == 0))
    return np.where(up, hi, lo)


def power_above(amax, top):
    """e8m0 bytes: the smallest power of two s >= 2^-126 with amax <= top s."""
    byte = np.ones(amax.shape, np.int64)
    while True:
        more = (amax > top * 2.0 ** (byte - 127.0)) & (byte < 254)
        if not more.any():
            return byte
        byte = byte + more


def quantise(x, fmt, exponent=0):
    """(codes, scale bytes) of a matrix [R, K], K filled up to whole blocks; scales as bytes [R, blocks]."""
    R, K = x.shape
    b = BLOCK[fmt]
    v = np.zeros((R, -(-K // b) * b))
    v[:, :K] = x
    v = v.reshape(R, -1, b)
    amax = np.abs(v).max(-1)
    finite = np.isfinite(amax)
    amax = np.where(finite, amax, 0.0)
    if fmt == E4M3:
        byte = nearest(amax * 2.0 ** -exponent / 6, E4M3_VALUES)
        s = E4M3_VALUES[byte] * 2.0 ** exponent
    else:
        byte = power_above(amax, 6.0)
        s = 2.0 ** (byte - 127.0)
    with np.errstate(all="ignore"):
        q = np.where(s[..., None] > 0, np.abs(v) / s[..., None], 0.0)
        codes = nearest(np.where(np.isfinite(q), q, 0.0), E2M1) + 8 * np.signbit(v)
    byte = np.where(finite, byte, 0x7f if fmt == E4M3 else 0xff)
    return codes.reshape(R, -1), byte


def scale_values(byte, fmt, exponent=0):
    if fmt == E8M0:
        return np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))
    return np.where(byte == 0x7f, np.nan, E4M3_VALUES[np.minimum(byte, 126)]) * 2.0 ** exponent


def values(codes, byte, fmt, exponent=0):
    """What a 4-bit matrix stands for."""
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    return v * np.repeat(scale_values(byte, fmt, exponent), BLOCK[fmt], 1)[:, :v.shape[1]]


def rounded(x, fmt, exponent=0):
    """x after the trip through 4 bits."""
    codes, byte = quantise(x, fmt, exponent)
    return values(codes, byte, fmt, exponent)[:, :x.shape[1]]


def pack(codes):
    """Two codes a byte, the even column low."""
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def tiles(byte):
    """Scale bytes [R, blocks] as they lie in memory: [row tiles, block tiles, 512]."""
    R, n = byte.shape
    out = np.zeros((-(-R // 128), -(-n // 4), 512), np.uint8)
    r, j = np.meshgrid(np.arange(R), np.arange(n), indexing="ij")
    out[r // 128, j // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + j % 4] = byte
    return out


def untile(t, R, n):
    r, j = np.meshgrid(np.arange(R), np.arange(n), indexing="ij")
    return t[r // 128, j // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + j % 4].astype(np.int64)


# ------------------------------------------------------------------ the optimiser's step
def adamw(p, g, m, v, lr, beta1, beta2, eps, decay, step):
    """(p, m, v) after a step, fp64."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p - lr * decay * p - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v


def _mix(x):
    x = ((x ^ (x >> 16)) * 0x243f6a89) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0xb7e15163) & 0xffffffff
    return x ^ (x >> 16)


def random_bits(first, n, seed, step):
    """The 32 bits of elements first .. first + n of a call."""
    key = _mix(_mix(_mix(seed & 0xffffffff) ^ (seed >> 32)) ^ step)
    i = np.arange(first, first + n, dtype=np.uint64)
    lo, hi = i & np.uint64(0xffffffff), i >> np.uint64(32)
    k = np.array([key if h == 0 else _mix(key ^ int(h)) for h in np.unique(hi)], np.uint64)[
        np.searchsorted(np.unique(hi), hi)]
    x = ((lo * np.uint64(0x9e3779b1)) & np.uint64(0xffffffff)) ^ k
    for shift, factor in ((16, 0x243f6a89), (15, 0xb7e15163)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def moment8_scales(x):
    """e8m0 bytes of a flat tensor of moments; 255 where a block has a value that is not finite."""
    v = np.zeros(-(-x.size // 32) * 32)
    v[:x.size] = x
    amax = np.abs(v.reshape(-1, 32)).max(1)
    return np.where(np.isfinite(amax), power_above(np.where(np.isfinite(amax), amax, 0.0), 448.0), 255)


def moment8_codes(x, byte, r16, floor):
    """e4m3 codes of x under the blocks' scales, rounded by 16 random bits each; floor: a value above zero is at
    least the smallest step."""
    finite = np.repeat(byte != 255, 32)[:x.size]
    y = np.where(finite, np.abs(x), 0.0) / np.repeat(2.0 ** (byte - 127.0), 32)[:x.size]
    lo = np.clip(np.searchsorted(E4M3_VALUES, y, side="right") - 1, 0, 125)
    share = (y - E4M3_VALUES[lo]) / (E4M3_VALUES[lo + 1] - E4M3_VALUES[lo])
    code = lo + (share >= 1.0 - (16.0 * r16 + 8.0) / 2.0 ** 20)
    if floor:
        code = np.where((y > 0) & (code == 0), 1, code)
    return np.where(finite, code | np.where(np.signbit(x), 128, 0), 0)


def moment8(x, r16, floor):
    """(codes, scale bytes) of a flat tensor of moments."""
    byte = moment8_scales(x)
    return moment8_codes(x, byte, r16, floor), byte


def values8(codes, byte):
    mag = E4M3_VALUES[np.minimum(codes & 127, 126)]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))
    return np.where(codes & 128, -mag, mag) * np.repeat(s, 32)[:codes.size]
