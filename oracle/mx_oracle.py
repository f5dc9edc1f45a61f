"""float64 oracle of the layer norm of include/norm.h and of include/mxfp4.h: numpy, from the formulas in the headers."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])     # of codes 0..7; 8..15: the negatives


def _per_row(v, M, other):
    """A sample's vectors [S, K], one for each of its rows."""
    return other if v is None else np.repeat(v, M // v.shape[0], 0)


def layer_rows(h, eps):
    """(n, r, nmax): the normed rows, the factor of each, and what bounds |n| before the mean is taken out."""
    mean = h.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    n = (h - mean) * r
    return n, r, np.abs(n) + r * np.abs(h).mean(1, keepdims=True)


def layer_fwd(h, w, b, scale, shift, eps):
    """(y, size): size bounds the terms that y is a sum of."""
    M = h.shape[0]
    n, _, nmax = layer_rows(h, eps)
    w, b = (1.0 if w is None else w), (0.0 if b is None else b)
    up, t = 1.0 + _per_row(scale, M, 0.0), _per_row(shift, M, 0.0)
    return (n * w + b) * up + t, (nmax * np.abs(w) + np.abs(b)) * np.abs(up) + np.abs(t)


def layer_bwd(dy, h, w, b, dh, res, gate, scale, eps, samples=1):
    """{name: (gradient, size of its terms)} of dx, dres, dw, dbias, dgate, dscale, dshift (the last three per sample)."""
    M, K = h.shape
    n, r, nmax = layer_rows(h, eps)
    w, b = (1.0 if w is None else w), (0.0 if b is None else b)
    up, gt = 1.0 + _per_row(scale, M, 0.0), _per_row(gate, M, 1.0)
    da = dy * up
    g = da * w
    dx = r * (g - g.mean(1, keepdims=True) - n * (g * n).mean(1, keepdims=True))
    size = r * (np.abs(g) + np.abs(g).mean(1, keepdims=True) + nmax * (np.abs(g) * nmax).mean(1, keepdims=True))
    if dh is not None:
        dx, size = dx + dh, size + np.abs(dh)
    per = lambda x: x.reshape(samples, M // samples, K).sum(1)
    out = {"dx": (dx, size), "dres": (dx * gt, size * np.abs(gt)),
           "dw": ((da * n).sum(0), (np.abs(da) * nmax).sum(0)), "dbias": (da.sum(0), np.abs(da).sum(0)),
           "dscale": (per(dy * (n * w + b)), per(np.abs(dy) * (nmax * np.abs(w) + np.abs(b)))),
           "dshift": (per(dy), per(np.abs(dy)))}
    if res is not None:
        out["dgate"] = (per(dx * res), per(size * np.abs(res)))
    return out


def quantize(x):
    """(codes [R, K] of 0..15, exponents [R, ceil(K / 32)]) of x [R, K]."""
    R, K = x.shape
    blocks = -(-K // 32)
    p = np.zeros((R, blocks * 32))
    p[:, :K] = x
    p = p.reshape(R, blocks, 32)
    bad = ~np.isfinite(p).all(2)
    p = np.where(bad[..., None], 0.0, p)
    top = np.abs(p).max(2)
    e = np.frexp(np.where(top > 0, top, 1.0))[1] - 1                 # floor(log2)
    E = np.where(top > 0, np.maximum(e - 2 + 127, 1), 1)
    v = np.abs(p) / np.ldexp(1.0, E - 127)[..., None]
    # the nearest value, a tie to the even code
    gap = np.abs(v[..., None] - VALUES)
    near = gap.min(-1, keepdims=True) == gap
    code = np.where(near, np.where(np.arange(8) % 2 == 0, np.arange(8), np.arange(8) + 100), 1000).argmin(-1)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(p))
    return code.reshape(R, -1)[:, :K].astype(np.uint8), np.where(bad, 255, E).astype(np.uint8)


def dequantize(codes, exponents):
    """What codes [R, K] and exponents [R, ceil(K / 32)] stand for."""
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes & 7]
    e = np.repeat(exponents.astype(np.int64), 32, 1)[:, :codes.shape[1]]
    return np.where(e == 255, np.nan, np.ldexp(v, e - 127))


def plain(codes):
    """Codes [R, K] two to a byte, as mxfp4_pack takes them."""
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def codes_of(plain_codes):
    return np.stack((plain_codes & 15, plain_codes >> 4), 2).reshape(plain_codes.shape[0], -1)
