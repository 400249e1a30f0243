"""Plain numpy, float64, of the operators beside densify: the dropout mask, the lookup, 8-bit codes and their products.
Written from the definitions; shares nothing with the kernels."""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=7):
    """Philox4x32: counter (four arrays or numbers of 32 bits), key (two numbers) -> four uint64 arrays of 32-bit words."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & LOW, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(n, d, p, seed, offset, first_row=0):
    """[n, d] truth values: the elements of rows first_row .. first_row + n - 1 that are kept."""
    e = np.uint64(first_row) * np.uint64(d) + np.arange(n * d, dtype=np.uint64)
    g = e[::4] // np.uint64(4)
    offset %= 1 << 64
    w = philox([g & LOW, g >> np.uint64(32), offset & 0xFFFFFFFF, offset >> 32], (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack([np.broadcast_to(x, g.shape) for x in w], axis=1).reshape(n, d)
    return words >= np.uint64(int(np.floor(float(np.float32(p)) * 2.0 ** 32)))


def factor(p, scale=1.0):
    """What kept elements are multiplied by, as fp32 holds it."""
    return float(np.float32(float(np.float32(scale)) / (1.0 - float(np.float32(p)))))


def dropout(x, p, seed, offset, add=None, scale=1.0):
    y = np.where(kept(*x.shape, p, seed, offset), x.astype(np.float64) * factor(p, scale), 0.0)
    return y if add is None else y + add.astype(np.float64)


def lookup(ids, weight, scale, p, seed, offset, pos=None, pos_ids=None):
    x = np.zeros((len(ids), weight.shape[1]))
    ok = (ids >= 0) & (ids < len(weight))
    x[ok] = weight[ids[ok]].astype(np.float64) * float(np.float32(scale))
    if pos is not None:
        ok = (pos_ids >= 0) & (pos_ids < len(pos))
        x[ok] += pos[pos_ids[ok]]
    return dropout(x, p, seed, offset)


# ---- 8-bit codes: (mantissa bits, exponent bias, largest)
FORMATS = {0: (3, 7, 448.0), 1: (2, 15, 57344.0)}


def decode(fmt):
    """The 256 values of a format."""
    m, bias, top = FORMATS[fmt]
    code = np.arange(256)
    sign, e, f = np.where(code >> 7, -1.0, 1.0), (code & 0x7F) >> m, (code & ((1 << m) - 1)) / 2.0 ** m
    v = sign * np.where(e == 0, f * 2.0 ** (1 - bias), (1 + f) * 2.0 ** (e - bias))
    if fmt == 0:
        v[[0x7F, 0xFF]] = np.nan
    else:
        v[0x7C], v[0xFC] = np.inf, -np.inf
        v[0x7D:0x80] = v[0xFD:] = np.nan
    return v


def encode(x, fmt):
    """Nearest codes, ties to the even code; x is at most the largest value in size, or no finite number."""
    v = decode(fmt)
    last = int(np.flatnonzero(v == FORMATS[fmt][2])[0])
    grid = v[:last + 1]
    a = np.abs(np.asarray(x, dtype=np.float64))
    fine = np.isfinite(a)
    a0 = np.where(fine, a, 0.0)
    assert (a0 <= grid[-1]).all()
    hi = np.searchsorted(grid, a0)
    lo = np.maximum(hi - 1, 0)
    down, up = a0 - grid[lo], grid[hi] - a0
    code = np.where(a0 == grid[hi], hi, np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi))
    code = np.where(fine, code, 0x7F if fmt == 0 else np.where(np.isinf(a), 0x7C, 0x7F))
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def quantize(x, fmt):
    """(codes [rows, K rounded up to 128], scales [rows, blocks rounded up to 4]) of x [rows, K]; NaN codes may differ."""
    rows, K = x.shape
    blocks = -(-K // 128)
    full = np.zeros((rows, blocks * 128))
    full[:, :K] = x
    part = full.reshape(rows, blocks, 128)
    most = np.where(np.isfinite(part), np.abs(part), 0.0).max(axis=2, initial=0.0)
    top = FORMATS[fmt][2]
    m, e = np.frexp(most / top)                                      # most / top = m 2^e, m in [0.5, 1)
    e = np.where(most == 0, -127, np.where(m == 0.5, e - 1, e))
    # the quotient may have been rounded to a power of two
    e = np.where(most > top * np.ldexp(1.0, e), e + 1, e)
    e = np.maximum(e, -127)
    codes = encode(part * np.ldexp(1.0, -e)[:, :, None], fmt).reshape(rows, blocks * 128)
    scales = np.zeros((rows, -(-blocks // 4) * 4), dtype=np.uint8)
    scales[:, :blocks] = e + 127
    return codes, scales


def values(codes, scales, fmt):
    rows, k = codes.shape
    e = scales[:, :k // 128].astype(np.int64) - 127
    return (decode(fmt)[codes].reshape(rows, -1, 128) * np.ldexp(1.0, e)[:, :, None]).reshape(rows, k)


def matmul(a, a_scales, fa, b, b_scales, fb, c_in=None):
    """(product, sum of the terms' magnitudes), [M, N] float64."""
    u, v = values(a, a_scales, fa), values(b, b_scales, fb)
    y, size = u @ v.T, np.abs(u) @ np.abs(v).T
    return (y, size) if c_in is None else (y + c_in, size + np.abs(c_in))
