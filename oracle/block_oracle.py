"""float64 oracle of the operators between attention and Linear layers (include/rope.h, include/norm.h,
include/xattn.h, the norm of include/w8a8.h): numpy, from the formulas in the headers."""
import numpy as np

D = 128


def pair_channels(pairing):
    """Channels (lo, hi) of the 64 pairs of a head."""
    j = np.arange(D // 2)
    return (2 * j, 2 * j + 1) if pairing == "interleaved" else (j, j + D // 2)


def angles(positions, pairs, theta):
    """[..., 64] radians for positions [..., 3] (reduced modulo a turn in extended precision)."""
    out, turn = [], 2 * np.longdouble("3.14159265358979323846264338327950288")
    for axis, n in enumerate(pairs):
        for i in range(n):
            freq = np.longdouble(theta[axis]) ** (-np.longdouble(i) / n)
            out.append(np.fmod(positions[..., axis].astype(np.longdouble) * freq, turn).astype(np.float64))
    return np.stack(out, -1)


def rotate(x, ang, pairing):
    """x [..., 128] turned by ang [..., 64]."""
    lo, hi = pair_channels(pairing)
    y = np.empty_like(x)
    y[..., lo] = x[..., lo] * np.cos(ang) - x[..., hi] * np.sin(ang)
    y[..., hi] = x[..., lo] * np.sin(ang) + x[..., hi] * np.cos(ang)
    return y


def _rope_norm(x, weight, norm, eps):
    """(r, w) broadcastable to x [B, H, N, d]."""
    if norm == "none":
        return 1.0, 1.0
    axes = (3,) if norm == "head" else (1, 3)
    r = 1.0 / np.sqrt((x * x).mean(axes, keepdims=True) + eps)
    if weight is None:
        return r, 1.0
    return r, weight.reshape(1, 1, 1, D) if norm == "head" else weight.reshape(1, x.shape[1], 1, D)


def rope_fwd(x, ang, pairing, weight=None, norm="none", eps=1e-6):
    """x [B, H, N, d], ang [B, N, 64]."""
    r, w = _rope_norm(x, weight, norm, eps)
    return rotate(x * r * w, ang[:, None], pairing)


def rope_bwd(dy, x, ang, pairing, weight=None, norm="none", eps=1e-6):
    """(dx, dw or None, scale): scale bounds the terms that dx is a difference of."""
    g = rotate(dy, -ang[:, None], pairing)
    lo, hi = pair_channels(pairing)
    size = np.empty_like(g)
    size[..., lo] = size[..., hi] = np.abs(dy[..., lo]) + np.abs(dy[..., hi])
    if norm == "none":
        return g, None, size
    r, w = _rope_norm(x, weight, norm, eps)
    axes = (3,) if norm == "head" else (1, 3)
    dx = r * w * g - x * r ** 3 * (x * w * g).mean(axes, keepdims=True)
    dw = (g * x * r).sum((0, 1, 2) if norm == "head" else (0, 2)).reshape(-1)
    scale = r * np.abs(w) * size + np.abs(x) * r ** 3 * (np.abs(x) * np.abs(w) * size).mean(axes, keepdims=True)
    return dx, dw, scale


def norm_fwd(h, w, eps):
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h * r * (1.0 if w is None else w)


def norm_bwd(dy, h, w, dh, eps):
    """(dx, dw, scale of the terms of dx)"""
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    g = dy if w is None else dy * w
    dx = r * g - h * r ** 3 * (h * g).mean(1, keepdims=True)
    scale = r * np.abs(g) + np.abs(h) * r ** 3 * np.abs(h * g).mean(1, keepdims=True)
    if dh is not None:
        dx, scale = dx + dh, scale + np.abs(dh)
    return dx, (dy * h * r).sum(0), scale


def xattn_fwd(q, k, v, lens=None, scale=None):
    """(out [B, H, Nq, d], lse [B, H, Nq]) for q [B, H, Nq, d], k and v [B, G, Nk, d]; a sample without keys: zeros, -inf."""
    B, H, Nq, d = q.shape
    G, Nk = k.shape[1], k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out, lse = np.zeros((B, H, Nq, d)), np.full((B, H, Nq), -np.inf)
    for b in range(B):
        n = Nk if lens is None else min(max(int(lens[b]), 0), Nk)
        if n == 0:
            continue
        for h in range(H):
            g = h // (H // G)
            s = q[b, h] @ k[b, g, :n].T * scale
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            l = p.sum(1, keepdims=True)
            out[b, h] = p / l @ v[b, g, :n]
            lse[b, h] = (m + np.log(l))[:, 0]
    return out, lse


def xattn_bwd(q, k, v, dout, lens=None, scale=None):
    """(dq, dk, dv)"""
    B, H, Nq, d = q.shape
    G, Nk = k.shape[1], k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        n = Nk if lens is None else min(max(int(lens[b]), 0), Nk)
        if n == 0:
            continue
        for h in range(H):
            g = h // (H // G)
            s = q[b, h] @ k[b, g, :n].T * scale
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            dp = dout[b, h] @ v[b, g, :n].T
            ds = p * (dp - (p * dp).sum(1, keepdims=True)) * scale
            dq[b, h] = ds @ k[b, g, :n]
            dk[b, g, :n] += ds.T @ q[b, h]
            dv[b, g, :n] += p.T @ dout[b, h]
    return dq, dk, dv
