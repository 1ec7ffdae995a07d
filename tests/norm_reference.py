"""Dropout from a counter, residual and layer norm in 64 bits (numpy), from their definitions, with bounds of the kernels' roundings."""
import numpy as np

F32 = 2.0 ** -24


def philox(block, site, step, seed):
    """Philox4x32-10 of the paper (Salmon et al., SC 2011) in Python's whole numbers."""
    mask = 0xFFFFFFFF
    c = [block & mask, site & mask, step & mask, (step >> 32) & mask]
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k0, b & mask, (a >> 32) ^ c[3] ^ k1, a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c


def factors(n, p, seed, step, site):
    t = int(p * 65536 + 0.5)
    if t == 0:
        return np.ones(n)
    mask = np.uint64(0xFFFFFFFF)
    g = np.arange((n + 7) // 8, dtype=np.uint64)
    full = lambda v: np.full_like(g, v & 0xFFFFFFFF)  # noqa: E731
    c = [g, full(site), full(step), full(step >> 32)]
    k0, k1, s32 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF, np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k0), b & mask, (a >> s32) ^ c[3] ^ np.uint64(k1), a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack(c, -1)
    u = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(-1)[:n]
    return np.where(u >= t, 65536 / (65536 - t), 0.0)


def dropout_add(y, x, f, u):
    """(value, bound)"""
    x = np.zeros_like(y) if x is None else x
    out = x + y * f
    return out, u * np.abs(out) * (1 + 8 * F32) + 3 * F32 * (np.abs(x) + np.abs(y * f))


def forward(x, y, w, b, eps, f, u):
    """{name: (value, bound)} of h, n, mean, rstd; x, y [rows][width]"""
    width = x.shape[1]
    yf = np.zeros_like(x) if y is None else y * f
    h = x + yf
    mean = h.mean(1, keepdims=True)
    c = h - mean
    rstd = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    b = np.zeros(width) if b is None else b
    n = c * rstd * w + b
    e_h = 3 * F32 * (np.abs(x) + np.abs(yf))
    e_mean = e_h.mean(1, keepdims=True) + F32 * (width + 4) * np.abs(h).mean(1, keepdims=True)
    e_c = e_h + e_mean + F32 * np.abs(c)
    # the variance's first-order error vanishes where the mean's does (sum c = 0); e_c^2 is what a shifted mean adds
    e_r = rstd * (((np.abs(c) * e_c).mean(1, keepdims=True) + (e_c * e_c).mean(1, keepdims=True)) * rstd ** 2 + F32 * (width + 12))
    e_n = np.abs(w) * (rstd * e_c + np.abs(c) * e_r + 4 * F32 * np.abs(c) * rstd) + 2 * F32 * (np.abs(n) + np.abs(b))
    return {"h": (h, u * np.abs(h) * (1 + 8 * F32) + e_h), "n": (n, u * (np.abs(n) + e_n) + e_n), "mean": (mean[:, 0], e_mean[:, 0] + F32 * np.abs(mean[:, 0])),
            "rstd": (rstd[:, 0], e_r[:, 0] + 4 * F32 * rstd[:, 0])}


def backward(dn, dh, h, w, mean, rstd, f, u, u_w):
    """{name: (value, bound)} of dx, dy, dw, db; mean, rstd [rows]: what the call is given"""
    rows, width = h.shape
    dh = np.zeros_like(h) if dh is None else dh
    mean, rstd = mean[:, None], rstd[:, None]
    hat = (h - mean) * rstd
    g = dn * w
    s0, s1 = g.mean(1, keepdims=True), (g * hat).mean(1, keepdims=True)
    dx = dh + rstd * (g - s0 - hat * s1)
    e_hat = 2 * F32 * (np.abs(hat) + np.abs(h * rstd) + np.abs(mean * rstd))
    e0 = F32 * (width + 4) * np.abs(g).mean(1, keepdims=True)
    e1 = F32 * (width + 6) * np.abs(g * hat).mean(1, keepdims=True) + (np.abs(g) * e_hat).mean(1, keepdims=True)
    e = np.abs(rstd) * (6 * F32 * (np.abs(g) + np.abs(s0) + np.abs(hat * s1)) + e0 + np.abs(hat) * e1 + e_hat * np.abs(s1)) + 2 * F32 * (np.abs(dh) + np.abs(dx))
    dw, db = (dn * hat).sum(0), dn.sum(0)
    e_w = F32 * (rows + 8) * np.abs(dn * hat).sum(0) + (np.abs(dn) * e_hat).sum(0)
    e_b = F32 * (rows + 8) * np.abs(dn).sum(0)
    return {"dx": (dx, e + u * (np.abs(dx) + e)), "dy": (dx * f, f * (e + u * (np.abs(dx) + e) + 3 * F32 * np.abs(dx))),
            "dw": (dw, e_w + u_w * (np.abs(dw) + e_w)), "db": (db, e_b + u_w * (np.abs(db) + e_b))}
