"""Block-scaled 8- and 4-bit values in numpy, 64 bits: codes, quantisers, and the operators that use them.

A value is a code times 2^(b - 127), b the scale byte of its block of 32 consecutive values of a row (255: NaN).
8-bit codes are E4M3 (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff are NaN), 4-bit codes E2M1.
"""
import numpy as np

BLOCK, STEP = 32, 128


def _decode(code, exp_bits, man_bits, bias):
    sign = (code >> (exp_bits + man_bits)) & 1
    e = (code >> man_bits) & ((1 << exp_bits) - 1)
    m = code & ((1 << man_bits) - 1)
    v = m * 2.0 ** (1 - bias - man_bits) if e == 0 else (1 + m / (1 << man_bits)) * 2.0 ** (e - bias)
    return -v if sign else v


E4M3 = np.array([np.nan if c & 0x7f == 0x7f else _decode(c, 4, 3, 7) for c in range(256)])
E2M1 = np.array([_decode(c, 2, 1, 1) for c in range(16)])
TOP = {8: 448.0, 4: 6.0}
_POSITIVE = {8: E4M3[:127], 4: E2M1[:8]}


def padded(K):
    return -(-K // STEP) * STEP


def _round(v, bits):
    """Codes of the nearest numbers, ties to the even code; |v| <= TOP."""
    grid = _POSITIVE[bits]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(grid, a, side="left"), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return pick + np.where(np.signbit(v), 128 if bits == 8 else 8, 0)


def quantize(x, bits):
    """Rows [rows, K] -> (codes [rows, Kp], scale bytes [rows, Kp / 32]), one code per element."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    x = np.pad(x, ((0, 0), (0, padded(K) - K))).reshape(rows, -1, BLOCK)
    amax = np.abs(x).max(axis=-1)
    finite = np.isfinite(amax)
    b = np.zeros(amax.shape, dtype=np.int64)
    # the smallest byte whose scale leaves no value above the largest code
    todo = finite & (amax > 0)
    e = np.zeros(amax.shape)
    e[todo] = np.ceil(np.log2(amax[todo] / TOP[bits]))
    e = np.where(todo & (amax > TOP[bits] * 2.0 ** e), e + 1, e)
    e = np.where(todo & (amax <= TOP[bits] * 2.0 ** (e - 1)), e - 1, e)
    b[todo] = np.clip(e[todo], -127, 127).astype(np.int64) + 127
    b[~finite] = 255
    v = np.where(finite[..., None], x, 0.0) / 2.0 ** (np.where(finite, b, 127) - 127.0)[..., None]
    codes = _round(v, bits)
    codes[~finite] = 0x7f if bits == 8 else 0
    return codes.reshape(rows, -1).astype(np.uint8), b.astype(np.uint8)


def dequantize(codes, scales, bits, K=None):
    table = E4M3 if bits == 8 else E2M1
    b = scales.astype(np.float64)
    s = np.where(b == 255, np.nan, 2.0 ** (b - 127))
    v = (table[codes].reshape(codes.shape[0], -1, BLOCK) * s[..., None]).reshape(codes.shape[0], -1)
    return v if K is None else v[:, :K]


def requantized(x, bits=8):
    """What x stands for after a trip through the format."""
    x = np.asarray(x, dtype=np.float64)
    return dequantize(*quantize(x, bits), bits, x.shape[1])


def pack_weight(codes, scales, bits):
    """Device-native bytes of a matrix whose codes [rows, Kp] and scales [rows, Kp / 32] are given: tiles of 16 rows x 128
    columns; 4 bits: lane l = 16 g + r holds columns 32 g .. of row r, even column in the low nibble; 8 bits: two halves,
    lane l holds columns 64 h + 16 g ..; scales: byte j of dword (tile row, 4-tile group, lane) belongs to tile 4 kg + j."""
    rows, Kp = codes.shape
    rt, KT = (rows + 31) // 32 * 2, Kp // STEP
    KG = (KT + 3) // 4
    c = np.zeros((rt * 16, Kp), dtype=np.uint8)
    c[:rows] = codes
    s = np.zeros((rt * 16, KG * 16), dtype=np.uint8)
    s[:rows, :Kp // BLOCK] = scales
    c = c.reshape(rt, 16, KT, STEP)
    if bits == 4:
        b = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(rt, 16, KT, 4, 16)      # row, tile, g, 16 bytes
        out = b.transpose(0, 2, 3, 1, 4)                                         # tile, g, row, bytes
    else:
        b = c.reshape(rt, 16, KT, 2, 4, 16)                                      # row, tile, half, g, 16 bytes
        out = b.transpose(0, 2, 3, 4, 1, 5)
    sc = s.reshape(rt, 16, KG, 4, 4).transpose(0, 2, 4, 1, 3)                    # (row, kg, j, g) -> kg, g, row, j
    return np.ascontiguousarray(out).reshape(-1), np.ascontiguousarray(sc).reshape(-1)


def add_rmsnorm(h, delta, weight, eps):
    s = h if delta is None else h + delta
    with np.errstate(divide="ignore", invalid="ignore"):
        x = s / np.sqrt((s * s).mean(axis=-1, keepdims=True) + eps)
    return s, x if weight is None else x * weight


def expert(x, w1, w3, w2):
    """One SwiGLU expert with 8-bit rows between its products; matrices as numbers."""
    a = x @ w1.T
    with np.errstate(over="ignore"):
        h = a / (1 + np.exp(-a)) * (x @ w3.T)
    return requantized(h) @ w2.T


def largest_flip(x, w1, w3, w2):
    """By row: the 2-norm that the output moves by if the value of h that counts most is rounded to the code beside its
    own (a step of E4M3 is at most 2^-3 of the value)."""
    a = x @ w1.T
    with np.errstate(over="ignore"):
        h = a / (1 + np.exp(-a)) * (x @ w3.T)
    return (np.abs(h) * np.linalg.norm(w2, axis=0)).max(axis=1) * 2.0 ** -3


def moe_ffn(x, ids, w, experts, shared=(), gate=None, expert=expert):
    """x [N, H] numbers of the 8-bit rows; experts: id -> (w1, w3, w2), absent ones contribute nothing."""
    N, H = x.shape
    y = np.zeros((N, H))
    for e in np.unique(ids):
        if int(e) not in experts:
            continue
        t, j = np.nonzero(ids == e)
        np.add.at(y, t, expert(x[t], *experts[int(e)]) * w[t, j][:, None])
    g = np.ones(N) if gate is None else 1 / (1 + np.exp(-(x @ gate)))
    for m in shared:
        y += g[:, None] * expert(x, *m)
    return y
