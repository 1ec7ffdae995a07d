"""Embeddings, the gated feed-forward block and the norms around a block in 64 bits (numpy), from their definitions, each value with a bound
of the kernels' roundings: {name: (value, bound)}.  u: half a step of the type that a result is rounded to."""
import math

import numpy as np

F32 = 2.0 ** -24
erf = np.vectorize(math.erf, otypes=[float])


# ---- embeddings ------------------------------------------------------------------------------------------------------
def embed(ids, table, scale, u):
    out = np.zeros((*ids.shape, table.shape[1]))
    real = (ids >= 0) & (ids < len(table))
    out[real] = table[ids[real]] * scale
    return out, (u * (1 + 4 * F32) + 2 * F32) * np.abs(out)


def embed_grad(d_out, ids, vocab, scale, u, old=None):
    """A sum of n values of 32 bits in any order is off by at most (n - 1) 2^-24 of the sum of their sizes; the scale, the sum with what
    stands there and the last rounding follow."""
    width = d_out.shape[-1]
    grad, size, count = np.zeros((vocab, width)), np.zeros((vocab, width)), np.zeros((vocab, 1))
    for i, row in zip(ids.reshape(-1), d_out.reshape(-1, width)):
        if 0 <= i < vocab:
            grad[i] += row * scale
            size[i] += np.abs(row * scale)
            count[i] += 1
    e = F32 * (count + 2) * size
    if old is not None:
        grad, e = grad + old, e + np.where(count > 0, 2 * F32 * (size + np.abs(old)), 0)
    return grad, np.where(count > 0, e + u * (np.abs(grad) + e), 0)


# ---- gated feed-forward block ---------------------------------------------------------------------------------------------
def act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        cdf = 0.5 * (1 + erf(g / math.sqrt(2)))
        return g * cdf, cdf + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    t = np.tanh(z)
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)


def product(a, b, e_a=0.0, e_b=0.0):
    """a b^T of values that are off by e_a and e_b: with sums in 32 bits"""
    c, size = a @ b.T, np.abs(a) @ np.abs(b).T
    e = F32 * (a.shape[1] + 4) * size
    if np.any(e_a):
        e = e + e_a @ np.abs(b).T
    if np.any(e_b):
        e = e + np.abs(a) @ e_b.T
    return c, e


def ffn_inner(x, wg, wu, name, u):
    """What the forward keeps.  The activation's derivative is at most 1.13, the derivative's 0.8.  In 32 bits exp(z) is off by 2^-24 (|z| + 2) of itself (its
    argument is rounded): the sigmoid by 2^-24 (|z| + 6) of itself and of what it lacks to 1.  Of z = 2 sqrt(2 / pi) (g + ..) a further three roundings; where
    |z| is large the factor that carries them is small, and |z| exp(-|z|) and z^2 exp(-|z|) stay below 0.6, which leaves 16 2^-24 of the value, and of the
    slope 16 2^-24 (1 + |g|).  erf is off by 4 2^-24 of 1."""
    g, eg = product(x, wg)
    up, eu = product(x, wu)
    a, slope = act(g, name)
    ea = 1.2 * eg + 16 * F32 * np.abs(g)
    es = eg + 16 * F32 * (1 + np.abs(g))
    out = {"by_gate": (up * slope, eu * np.abs(slope) + (np.abs(up) + eu) * es), "by_up": (a, ea), "hidden": (a * up, eu * np.abs(a) + (np.abs(up) + eu) * ea)}
    return {k: (v, (e + F32 * np.abs(v)) * (1 + u) + u * np.abs(v)) for k, (v, e) in out.items()}


def ffn_out(hidden, wd, u):
    y, e = product(hidden, wd)
    return y, e * (1 + u) + u * np.abs(y)


def ffn_grads(dy, x, wg, wu, wd, by_gate, by_up, hidden, u):
    """From what the forward kept.  dG and dU are rounded before their products."""
    dh, eh = product(dy, np.ascontiguousarray(wd.T))
    dg, du = dh * by_gate, dh * by_up
    eg, eu = (np.abs(p) * (eh + F32 * np.abs(dh)) * (1 + u) + u * np.abs(dh * p) for p in (by_gate, by_up))
    dx1, e1 = product(np.hstack([dg, du]), np.hstack([wg.T, wu.T]), np.hstack([eg, eu]))
    out = {"dx": (dx1, e1), "dw_gate": product(dg.T, x.T, eg.T), "dw_up": product(du.T, x.T, eu.T), "dw_down": product(dy.T, hidden.T)}
    return {k: (v, e * (1 + u) + u * np.abs(v)) for k, (v, e) in out.items()}


# ---- norms around a block --------------------------------------------------------------------------------------------------
def _norm(v, e_v, eps, rms):
    """hat, mean, rstd of rows that are off by e_v, with bounds"""
    width = v.shape[1]
    mean = np.zeros((len(v), 1)) if rms else v.mean(1, keepdims=True)
    e_mean = 0 * mean if rms else e_v.mean(1, keepdims=True) + F32 * (width + 4) * np.abs(v).mean(1, keepdims=True)
    c = v - mean
    e_c = e_v + e_mean + F32 * np.abs(c)
    rstd = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    e_r = rstd * (((np.abs(c) * e_c).mean(1, keepdims=True) + (e_c * e_c).mean(1, keepdims=True)) * rstd ** 2 + F32 * (width + 12))
    hat = c * rstd
    return hat, rstd * e_c + np.abs(c) * e_r + 2 * F32 * np.abs(hat), (mean, e_mean + F32 * np.abs(mean)), (rstd, e_r + 4 * F32 * rstd)


def gate_norm(x, y, wp, bp, gate, w, b, scale, eps, rms, u):
    hat, e_hat, m0, r0 = _norm(y, np.zeros_like(y), eps, rms)
    c = hat * wp + bp
    e_c = np.abs(wp) * e_hat + 2 * F32 * (np.abs(hat * wp) + np.abs(bp))
    h = scale * x + gate * c
    e_h = np.abs(gate) * e_c + 3 * F32 * (np.abs(scale * x) + np.abs(gate * c))
    hat, e_hat, m1, r1 = _norm(h, e_h, eps, rms)
    n = hat * w + b
    e_n = np.abs(w) * e_hat + 2 * F32 * (np.abs(hat * w) + np.abs(b))
    stats = tuple(np.stack([p[i][:, 0] for p in (m0, r0, m1, r1)]) for i in range(2))
    return {"h": (h, u * (np.abs(h) + e_h) + e_h), "n": (n, u * (np.abs(n) + e_n) + e_n), "stats": stats}


def _norm_grad(g, e_g, v, mean, rstd, rms):
    """The gradient of v from that of hat, where hat is made of the given statistics"""
    width = v.shape[1]
    hat = (v - mean) * rstd
    e_hat = 2 * F32 * (np.abs(hat) + np.abs(v * rstd) + np.abs(mean * rstd))
    s0 = 0 * mean if rms else g.mean(1, keepdims=True)
    s1 = (g * hat).mean(1, keepdims=True)
    e0 = 0 * mean if rms else F32 * (width + 4) * np.abs(g).mean(1, keepdims=True) + e_g.mean(1, keepdims=True)
    e1 = F32 * (width + 6) * np.abs(g * hat).mean(1, keepdims=True) + (np.abs(g) * e_hat + e_g * (np.abs(hat) + e_hat)).mean(1, keepdims=True)
    d = rstd * (g - s0 - hat * s1)
    e = np.abs(rstd) * (6 * F32 * (np.abs(g) + np.abs(s0) + np.abs(hat * s1)) + e_g + e0 + (np.abs(hat) + e_hat) * e1 + e_hat * np.abs(s1))
    return d, e, hat, e_hat


def gate_norm_grads(dn, dh, h, y, stats, wp, bp, gate, w, scale, rms, u, u_w):
    """From the h and the statistics that the call is given"""
    rows = len(h)
    m0, r0, m1, r1 = (s[:, None] for s in stats)
    g = dn * w
    d, e, hhat, e_hhat = _norm_grad(g, F32 * np.abs(g), h, m1, r1, rms)
    dht = dh + d
    e = e + 2 * F32 * (np.abs(dh) + np.abs(dht))
    g = dht * (gate * wp)
    dy, e_y, yhat, e_yhat = _norm_grad(g, np.abs(gate * wp) * e + 3 * F32 * np.abs(g), y, m0, r0, rms)
    dx = scale * dht

    def column(v, e_v):
        """the sum over the rows and its bound"""
        return v.sum(0), F32 * (rows + 8) * np.abs(v).sum(0) + e_v.sum(0)

    (A, eA), (B, eB) = column(dht * yhat, np.abs(dht) * e_yhat + e * (np.abs(yhat) + e_yhat)), column(dht, e)
    out = {"dpost_weight": (gate * A, np.abs(gate) * eA + F32 * np.abs(gate * A)), "dpost_bias": (gate * B, np.abs(gate) * eB + F32 * np.abs(gate * B)),
           "dgate": (wp * A + bp * B, np.abs(wp) * eA + np.abs(bp) * eB + 2 * F32 * (np.abs(wp * A) + np.abs(bp * B))),
           "dweight": column(dn * hhat, np.abs(dn) * e_hhat + F32 * np.abs(dn * hhat)), "dbias": column(dn, 0 * dn)}
    out = {k: (v, e_v + u_w * (np.abs(v) + e_v)) for k, (v, e_v) in out.items()}
    e_x = np.abs(scale) * e + F32 * np.abs(dx)
    out.update(dx=(dx, e_x + u * (np.abs(dx) + e_x)), dy=(dy, e_y + u * (np.abs(dy) + e_y)))
    return out
