"""The inner step's operators in 64 bits, from their definitions (numpy), for the tests."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_reference(x):
    """(codes, scale bytes, values) of the rows of x (64 bits) in blocks of 32; codes and bytes of NaN blocks are 0 and 255."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    ok = np.isfinite(b).all(-1)
    safe = np.where(ok[..., None], b, 0.0)
    top = np.abs(safe).max(-1)
    X = np.zeros((rows, nb), np.int64)                       # the smallest X with top <= 6 * 2^(X - 127)
    for e in range(0, 254):
        X = np.where(top > 6.0 * 2.0 ** (e - 127), e + 1, X)
    y = safe / (2.0 ** (X - 127.0))[..., None]
    dist = np.abs(np.abs(y)[..., None] - GRID)
    best = dist.min(-1, keepdims=True)
    at = dist == best
    first = at.argmax(-1)
    last = 7 - at[..., ::-1].argmax(-1)
    code = np.where((first == last) | (first % 2 == 0), first, last)     # a tie goes to the even code
    values = np.copysign(GRID[code], safe) * (2.0 ** (X - 127.0))[..., None]
    code = code + 8 * np.signbit(safe)
    values[~ok] = np.nan
    code[~ok] = 0
    X[~ok] = 255
    return code.reshape(rows, -1), X, values.reshape(rows, -1)[:, :cols]


def mx4_layout(buf, rows, cols):
    """(codes, scale bytes) of a 4-bit matrix as the header lays it out, tiles' padding included."""
    buf = np.asarray(buf, np.uint8)
    rt, kt = -(-rows // 32), -(-cols // 128)
    tiles = buf[:rt * kt * 2048].reshape(rt, kt, 4, 32, 16)               # row tile, column tile, block, row, byte
    nib = np.stack([tiles & 15, tiles >> 4], -1).reshape(rt, kt, 4, 32, 32)
    codes = nib.transpose(0, 3, 1, 2, 4).reshape(rt * 32, kt * 128)
    st = -(-rows // 64)
    # scale tile, column tile, block % 2, row % 32, row / 32, block / 2
    sc = buf[rt * kt * 2048:rt * kt * 2048 + st * kt * 256].reshape(st, kt, 2, 32, 2, 2)
    scales = sc.transpose(0, 4, 3, 1, 5, 2).reshape(st * 64, kt * 4)
    return codes.astype(np.int64), scales.astype(np.int64)


def _pow2(e):
    return np.ldexp(1.0, np.asarray(e, np.int64))


def decode8(codes, scales, block_of, signed):
    """Values (64 bits) of 8-bit moments; block_of: block of each element."""
    c = codes.astype(np.int64)
    mag = c & 127 if signed else c
    exp, man = mag >> 3, mag & 7
    lowest = -14 if signed else -30
    x = np.where(exp == 0, man / 8.0 * _pow2(lowest), (1 + man / 8.0) * _pow2(exp - 1 + lowest))
    if signed:
        x = np.where(c > 127, -x, x)
    s = scales.astype(np.int64)[block_of]
    return np.where(s == 255, np.nan, np.where(s == 0, 0.0, x * _pow2(s - 127)))


def fmix32(h):
    h = np.asarray(h, np.uint64)
    h ^= h >> np.uint64(16)
    h = h * np.uint64(0x85EBCA6B) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(13)
    h = h * np.uint64(0xC2B2AE35) & np.uint64(0xFFFFFFFF)
    return h ^ (h >> np.uint64(16))


def random_bits(seed, block_of, place):
    return fmix32(fmix32(fmix32(seed) ^ block_of.astype(np.uint64)) ^ place.astype(np.uint64))


def encode8_positions(x, rnd, top, signed):
    """(X, where the value lies on the block's scale of codes counted from 0, random part added): the code is the integer part."""
    lowest = -14 if signed else -30
    X = np.ones(top.shape, np.int64)
    for e in range(1, 253):
        X = np.where(top > 1.875 * 2.0 ** (e - 127), e + 1, X)
    y = np.abs(x) / _pow2(X - 127)
    exp = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))).astype(np.int64), lowest)
    exp = np.where(y < _pow2(exp), np.maximum(exp - 1, lowest), np.where(y >= 2 * _pow2(exp), exp + 1, exp))
    at = (exp - lowest) * 8 + y / _pow2(exp) * 8              # subnormals count from 0, binades of 8 follow
    return X, at + (rnd + 0.5) / 65536.0


def adamw_reference(theta, grad, m, v, scale, keep, p):
    """New (theta, m, v) in 64 bits and bounds of the error of the fp32 computation, to first order: u = 2^-24 for every
    product, sum, quotient, root and rounded constant on the way."""
    u = 2.0 ** -24
    g = grad * scale
    m1 = p["beta1"] * m + (1 - p["beta1"]) * g
    v1 = p["beta2"] * v + (1 - p["beta2"]) * g * g
    em = 5 * u * (np.abs(p["beta1"] * m) + np.abs((1 - p["beta1"]) * g))      # constant, scale, product, sum (and one to spare)
    ev = 7 * u * v1                                                           # all terms positive; g enters squared
    r = 1 / np.sqrt(1 - p["beta2"] ** p["step"])
    rate = p["lr"] / (1 - p["beta1"] ** p["step"])
    den = np.sqrt(v1) * r + p["eps"]
    upd = rate * m1 / den
    rel_den = 3.5 * u + 5 * u                                                 # half of ev's, root, constant, product, constant, sum
    new = theta * keep - upd
    et = em * rate / den + np.abs(upd) * (rel_den + 4 * u) + 6 * u * np.abs(theta) + u * np.abs(new)
    return new, m1, v1, et + 2e-45, em + 2e-45, ev + 2e-45
