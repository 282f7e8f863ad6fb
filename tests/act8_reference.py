"""Plain 64-bit forms of the training operators around 8-bit activation checkpoints, for the
tests: written from the definitions in include/natcomp.h, numpy only."""
import numpy as np

BLOCK = 32


def pitch_of(cols):
    return -(-cols // BLOCK) * BLOCK


def stream_bytes(seed, worker, count, domain=6):
    """Bytes 0 .. count-1 of the Philox4x32-10 stream (seed, worker, domain)."""
    q = np.arange(-(-count // 16), dtype=np.uint64)
    m32 = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    c = [q & m32, q >> sh, np.full_like(q, worker), np.full_like(q, domain)]
    for r in range(10):
        k0 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ k0, b & m32, (a >> sh) ^ c[3] ^ k1, a & m32]
    return np.stack(c, 1).astype("<u4").reshape(-1).view(np.uint8)[:count]


def scale_bytes(x):
    """e + 127 of every block of the float64 rows x (rows, cols); 255 where not finite."""
    rows, cols = x.shape
    p = pitch_of(cols)
    b = np.zeros((rows, p))
    b[:, :cols] = x
    top = np.abs(b.reshape(rows, -1, BLOCK)).max(2)
    out = np.full(top.shape, 255, np.int64)
    ok = np.isfinite(top)
    e = np.full(top.shape, -118, np.int64)
    pos = ok & (top > 0)
    # smallest e with top <= 127 * 2^e
    guess = np.zeros(top.shape, np.int64)
    guess[pos] = np.floor(np.log2(top[pos] / 127)).astype(np.int64) - 1
    for _ in range(3):
        guess[pos] += top[pos] > np.ldexp(127.0, guess[pos])
    e[pos] = np.maximum(guess[pos], -118)
    out[ok] = e[ok] + 127
    return out.astype(np.uint8)


def encode(x, random=False, seed=0, worker=0):
    """codes (rows, pitch), scales (rows, pitch / 32) of the rows x."""
    x = np.asarray(x)
    neg = np.signbit(x)
    x = x.astype(np.float64)
    rows, cols = x.shape
    p = pitch_of(cols)
    scales = scale_bytes(x)
    b = np.zeros((rows, p))
    b[:, :cols] = x
    sign = np.zeros((rows, p), np.int64)
    sign[:, :cols] = neg
    s = np.repeat(scales, BLOCK, 1).astype(np.int64)
    bad = s == 255
    b[bad] = 0
    y = np.ldexp(np.abs(b), 127 - s)
    if random:
        fine = np.rint(y * 256).astype(np.int64)
        r = stream_bytes(seed, worker, rows * p).reshape(rows, p).astype(np.int64)
        m = (fine + r) >> 8
    else:
        m = np.rint(y).astype(np.int64)
    codes = np.where(bad, 0, m | (sign << 7))
    return codes.astype(np.uint8), scales


def decode(codes, scales, cols):
    c = np.asarray(codes).astype(np.int64)
    s = np.repeat(np.asarray(scales).astype(np.int64), BLOCK, 1)
    v = np.ldexp((c & 127).astype(np.float64), s - 127)
    v = np.where(c & 128, -v, v)
    v[s == 255] = np.nan
    return v[:, :cols]


def layer_norm(x, gamma, beta, eps):
    """y, mean, rstd, xh in float64; gamma, beta may be None."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(1) + eps)
    xh = d * rstd[:, None]
    y = xh * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean, rstd, xh


def layer_norm_backward(dy, xh, rstd, gamma, dres=None):
    """dx, dgamma, dbeta in float64."""
    dy = np.asarray(dy, np.float64)
    xh = np.asarray(xh, np.float64)
    g = dy * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    m1 = g.mean(1, keepdims=True)
    m2 = (g * xh).mean(1, keepdims=True)
    dx = np.asarray(rstd, np.float64)[:, None] * (g - m1 - xh * m2)
    if dres is not None:
        dx = dx + np.asarray(dres, np.float64)
    return dx, (dy * xh).sum(0), dy.sum(0)


def weight_grad(dy, xh, gamma, beta):
    """dw (n, k), db (n) in float64: the input of the layer is gamma * xh + beta."""
    dy = np.asarray(dy, np.float64)
    a = np.asarray(xh, np.float64)
    if gamma is not None:
        a = a * np.asarray(gamma, np.float64)
    if beta is not None:
        a = a + np.asarray(beta, np.float64)
    return dy.T @ a, dy.sum(0)
