"""Self-attention with a relative position bias in 64 bits on the CPU, written pair by pair from its definition, with what the kernels'
roundings can add up to at every output (``bound``).  Nothing here comes from the library."""
import math

import numpy as np


def t5_table(n_buckets, max_distance, both_ways):
    """T5's buckets in whole numbers: the range that begins with the j-th step begins at the first n with (n / e)^L >= (m / e)^j."""
    half = n_buckets // 2 if both_ways else n_buckets
    e = half // 2
    L = half - e
    first = list(range(e + 1))
    for j in range(1, L):
        n = first[-1]
        while n ** L < e ** (L - j) * max_distance ** j:
            n += 1
        first.append(n)
    out = np.zeros(2 * max_distance + 1, np.int32)
    for d in range(-max_distance, max_distance + 1):
        away = abs(d) if both_ways else max(-d, 0)
        out[d + max_distance] = sum(1 for f in first[1:] if f <= away) + (half if both_ways and d > 0 else 0)
    return out


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


class Reference:
    """q, d_o [B][H][nq][D], k, v [B][KV][nk][D] float64 arrays of values the device has exactly, bias [buckets][H], table
    [2M + 1], lengths and starts: lists or None."""

    def __init__(self, q, k, v, bias, table, scale, causal, lengths=None, starts=None, d_o=None, dtype="bf16", bias_dtype=None):
        B, H, nq, D = q.shape
        KV, nk = k.shape[1:3]
        M, nb = (len(table) - 1) // 2, bias.shape[0]
        G = H // KV
        u, f32 = half_step(dtype), 2.0 ** -24
        self.o, self.lse = np.zeros(q.shape), np.full((B, H, nq), -np.inf)
        self.o_bound, self.lse_bound = np.zeros(q.shape), np.zeros((B, H, nq))
        names = ("dq", "dk", "dv", "dbias")
        for name, like in zip(names, (q, k, v, bias)):
            setattr(self, name, np.zeros(like.shape))
            setattr(self, name + "_bound", np.zeros(like.shape))
        for b in range(B):
            n = nk if lengths is None else min(max(int(lengths[b]), 0), nk)
            s0 = 0 if starts is None else int(starts[b])
            rows = [i for i in range(nq) if 0 <= s0 + i < n]
            if not rows:
                continue
            pos = np.array([s0 + i for i in rows])
            key = np.arange(n)
            rel = key[None, :] - pos[:, None]
            bucket = np.clip(np.asarray(table)[np.clip(rel, -M, M) + M], 0, nb - 1)
            seen = rel <= 0 if causal else np.ones_like(rel, bool)
            for h in range(H):
                g = h // G
                Q, K, V = q[b, h, rows], k[b, g, :n], v[b, g, :n]
                with np.errstate(invalid="ignore"):
                    A = Q @ K.T * scale + bias[bucket, h]
                A = np.where(seen, A, -np.inf)
                top = A.max(1, keepdims=True)
                live = np.isfinite(top[:, 0])
                P = np.where(live[:, None], np.exp(A - np.where(np.isfinite(top), top, 0)), 0)
                total = P.sum(1, keepdims=True)
                P = P / np.where(total > 0, total, 1)
                lse = np.where(live, np.where(live, top[:, 0], 0) + np.log(np.where(total[:, 0] > 0, total[:, 0], 1)), -np.inf)
                O = P @ V
                self.o[b, h, rows], self.lse[b, h, rows] = O, lse
                # scores in fp32: D products and their sum, the bias joined, the exponent's constant; the exponential's own error
                fin = np.where(np.isfinite(A), np.abs(A), 0)
                es = f32 * ((D + 4) * (np.abs(Q) @ np.abs(K).T) * scale + 6 * fin + 6 * np.abs(np.where(live, lse, 0))[:, None] + 4)
                ep = (es + (P * es).sum(1, keepdims=True) + f32 * (n + 8)) * P      # of a probability
                e_o = u * (P @ np.abs(V)) + ep @ np.abs(V) + f32 * (n + 8) * (P @ np.abs(V))
                self.lse_bound[b, h, rows] = (P * es).sum(1) + es.max(1) * 1e-3 + f32 * (n + 8) + 2 * f32 * np.abs(np.where(live, lse, 0))
                e_o = e_o + u * (np.abs(O) + e_o)
                self.o_bound[b, h, rows] = e_o
                if d_o is None:
                    continue
                dO = np.where(live[:, None], d_o[b, h, rows], 0)
                dP = dO @ V.T
                delta = (dO * O).sum(1, keepdims=True)
                dS = P * (dP - delta)
                self.dq[b, h, rows] = dS @ K * scale
                self.dk[b, g, :n] += dS.T @ Q * scale
                self.dv[b, g, :n] += P.T @ dO
                e_delta = (np.abs(dO) * e_o).sum(1, keepdims=True) + f32 * (D + 4) * (np.abs(dO) * np.abs(O)).sum(1, keepdims=True)
                ep2 = ep + P * self.lse_bound[b, h, rows][:, None]  # the backward's P comes from the rounded LSE
                e_ds = ep2 * np.abs(dP - delta) + P * (e_delta + f32 * (D + 4) * (np.abs(dO) @ np.abs(V).T)) + 4 * f32 * np.abs(dS)
                e_op = e_ds + u * (np.abs(dS) + e_ds)  # as an operand
                self.dq_bound[b, h, rows] = (e_op + f32 * (n + 8) * np.abs(dS)) @ np.abs(K) * scale
                self.dk_bound[b, g, :n] += (e_op + f32 * (nq * G + 8) * np.abs(dS)).T @ np.abs(Q) * scale
                self.dv_bound[b, g, :n] += (ep2 + (u + f32 * (nq * G + 8)) * P).T @ np.abs(dO)
                for x in range(nb):
                    at = bucket == x
                    self.dbias[x, h] += dS[at].sum()
                    self.dbias_bound[x, h] += e_ds[at].sum() + f32 * (at.sum() + 64) * np.abs(dS[at]).sum()
        for name in ("dq", "dk", "dv", "dbias"):
            ru = half_step(bias_dtype or dtype) if name == "dbias" else u
            v_, b_ = getattr(self, name), getattr(self, name + "_bound")
            setattr(self, name + "_bound", b_ + ru * (np.abs(v_) + b_))


def check(got, want, bound, name):
    """Everywhere within its bound; infinities alike."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fin), f"{name}: finite where it should not be, or the other way round"
    assert np.array_equal(got[~fin], want[~fin]), name
    off, most = np.abs(got[fin] - want[fin]), (bound + 1e-30)[fin]
    if off.size:
        worst = float((off / most).max())
        assert worst <= 1.0, f"{name}: {worst:.3g} times its bound (largest difference {off.max():.3g})"
        return worst
    return 0.0
