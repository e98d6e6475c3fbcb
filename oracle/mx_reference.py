"""The block-scaled formats, the norm and the layer on a 4-bit backbone from their definitions, in numpy and 64 bits.
Blocks of 32 values along a row share the scale 2^(s - 127); s = 255 makes them NaN."""
import numpy as np

BLOCK = 32


def elements(fmt):
    """The value of every code of a format."""
    if fmt == "e2m1":
        half = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        return np.array(half + [-v for v in half])
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = np.nan if (c & 127) == 127 else v
        out[c] *= -1.0 if c & 128 else 1.0
    return out


def unpack(codes, fmt):
    """[rows, K] codes, one to an entry."""
    codes = np.asarray(codes, np.uint8)
    if fmt == "e4m3":
        return codes
    out = np.empty((codes.shape[0], 2 * codes.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out


def pack(one, fmt):
    return one if fmt == "e4m3" else (one[:, 0::2] | one[:, 1::2] << 4).astype(np.uint8)


def scale_values(scales):
    s = np.asarray(scales).astype(np.float64)
    return np.where(s == 255, np.nan, np.exp2(s - 127))


def dequantize(codes, scales, fmt):
    v = elements(fmt)[unpack(codes, fmt)]
    return v * np.repeat(scale_values(scales), BLOCK, axis=1)


def quantize(x, fmt):
    """(codes, scales) of [rows, K] values: brute force over the format's magnitudes, ties to the even code."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    table = elements(fmt)
    pos = table[:8] if fmt == "e2m1" else table[:127]
    b = x.reshape(rows, K // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(-1)
    amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1))
    e = np.full(amax.shape, -127)
    for k in range(-126, 128):  # the smallest exponent that leaves the largest value in range
        e = np.where((amax > pos[-1] * 2.0 ** (k - 1)) & (amax <= pos[-1] * 2.0 ** k), k, e)
    u = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(e)[..., None]
    code = np.searchsorted(pos, u)  # pos[code - 1] < u <= pos[code]
    code = np.minimum(code, len(pos) - 1)
    lower = np.maximum(code - 1, 0)
    down, up = u - pos[lower], pos[code] - u
    code = np.where((down < up) | ((down == up) & (lower % 2 == 0)), lower, code)
    code = np.where(np.signbit(b), code + (8 if fmt == "e2m1" else 128), code).astype(np.uint8)
    return pack(code.reshape(rows, K), fmt), np.where(bad, 255, e + 127).astype(np.uint8)


def rms_norm(x, gamma, eps, residual=None):
    """(h, y)."""
    h = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    return h, h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * np.asarray(gamma, np.float64)


def linear(Xb, W, X=None, row_adapter=None, A=(), B=(), scale=()):
    """(Y, S, D): the layer; for every output the sum of the magnitudes of all that is added up, and of the adapter term's rank products."""
    Y = Xb @ W.T
    S = np.abs(Xb) @ np.abs(W).T
    term = np.zeros_like(Y)
    if row_adapter is not None:
        for a in sorted(set(int(i) for i in row_adapter if i >= 0)):
            t = np.nonzero(np.asarray(row_adapter) == a)[0]
            V = X[t] @ A[a].T
            Y[t] += scale[a] * (V @ B[a].T)
            S[t] += scale[a] * (np.abs(X[t]) @ np.abs(A[a]).T @ np.abs(B[a]).T)
            term[t] = abs(scale[a]) * (np.abs(V) @ np.abs(B[a]).T)
    return Y, S, term
