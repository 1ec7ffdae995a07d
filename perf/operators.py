"""The operators around the hierarchical attention whose time counts: what a decoder layer calls, and the values it gets.

  attn   self-attention with a learned relative position bias by buckets: causal or in both directions, forward, forward and
         backward (the gradient of the bias among its results), and for new tokens at the end of a cache
  drop   dropout from a counter-based generator, added to a residual or by itself
  norm   residual + dropout + layer norm, forward, or forward and backward

Every operator stands here in its plain form too (elementary torch operations in 32 bits), and `exact` says what the definition
gives in 64 bits.  `own` selects between the plain forms and the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases --------------------------------------------------------------------------------------------------
def _attn(name, batch, heads, kv_heads, head_dim, n_q, n_kv, *, causal=True, ragged=False, at_end=False, dtype="bf16", buckets=32,
          distance=128, backward=False):
    case = dict(kind="attn", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, n_q=n_q, n_kv=n_kv, causal=causal,
                ragged=ragged, at_end=at_end, dtype=dtype, buckets=buckets, distance=distance, backward=backward)
    return dict(case, name=name) if name else case


def _drop(name, rows, width, p, *, residual, dtype="bf16"):
    case = dict(kind="drop", rows=rows, width=width, p=p, residual=residual, dtype=dtype)
    return dict(case, name=name) if name else case


def _norm(name, rows, width, p, *, backward, dtype="bf16"):
    case = dict(kind="norm", rows=rows, width=width, p=p, backward=backward, dtype=dtype)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one new token of one document in a decoder layer, where latency counts
        _attn("token-1000", 1, 12, 12, 64, 1, 1000, at_end=True),
        # a full serving batch, one new token each, caches of different lengths, four query heads to a key head
        _attn("tokens-8192-shared", 32, 16, 4, 128, 1, 8192, ragged=True, at_end=True),
        # a chunk of a prompt behind what the cache holds already
        _attn("chunk-200-of-4096", 4, 12, 12, 64, 200, 4096, ragged=True, at_end=True),
        # the decoder's own attention in a training step of the summarisation model
        _attn("train-512", 4, 12, 12, 64, 512, 512, backward=True),
        # one long prompt through a layer, forward only
        _attn("prompt-8192", 2, 12, 12, 64, 8192, 8192),
        # a long training step at head size 128
        _attn("train-4096-d128", 2, 16, 16, 128, 4096, 4096, backward=True),
        # both directions, a padded batch of odd length, as an encoder without a hierarchy trains
        _attn("train-2047-both-ways", 3, 12, 12, 64, 2047, 2047, causal=False, ragged=True, backward=True),
        # the path that checks a model's numbers
        _attn("check-f32-512", 1, 4, 2, 64, 512, 512, dtype="f32", backward=True),
        # dropout of the embeddings of one document in 32 bits
        _drop("drop-f32-1000", 1000, 768, 0.1, residual=False, dtype="f32"),
        # the end of a block: a batch of 4 x 8192 positions
        _drop("drop-add-32768", 32768, 768, 0.1, residual=True),
        # four new tokens between two layers, nothing dropped
        _norm("norm-tokens-4", 4, 768, 0.0, backward=False),
        # the block of a training step on 4 x 8192 positions
        _norm("norm-train-32768", 32768, 768, 0.1, backward=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["train", "train", "forward", "tokens", "tokens", "check", "drop", "norm", "norm"])
    if what == "drop":
        width = rng.choice([rng.randint(1, 1500), rng.choice([512, 768, 1024, 2048])])
        return _drop(None, _log_int(rng, 1, max(1, 25_000_000 // width)), width, rng.choice([0.1, 0.1, 0.25, 0.5]), residual=rng.random() < 0.6,
                     dtype=rng.choice(["bf16", "bf16", "f32"]))
    if what == "norm":
        width = rng.choice([rng.randint(2, 1500), rng.choice([512, 768, 1024, 2048])])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _norm(None, _log_int(rng, 1, max(1, (25_000_000 if dtype == "bf16" else 10_000_000) // width)), width, rng.choice([0.0, 0.1, 0.1, 0.3]),
                     backward=rng.random() < 0.6, dtype=dtype)
    d, kv = rng.choice([64, 64, 128]), rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 1, 2, 3, 4]) if kv < 12 else 12
    buckets, distance = rng.choice([(32, 128), (32, 128), (64, 512), (16, 40)])
    kinds = dict(buckets=buckets, distance=distance)
    if what == "tokens":
        n = _log_int(rng, 16, 32768)
        chunk = 1 if rng.random() < 0.6 else rng.randint(1, min(n, 256))
        most = max(1, min(128_000_000 // (kv * n * d), 200_000_000 // (heads * chunk * n)))
        return _attn(None, rng.randint(1, min(32, most)), heads, kv, d, chunk, n, ragged=rng.random() < 0.7 and n >= 2 * chunk, at_end=True, **kinds)
    if what == "check":
        n = _log_int(rng, 16, 1024)
        return _attn(None, rng.randint(1, 2), heads, kv, d, n, n, causal=rng.random() < 0.6, ragged=rng.random() < 0.5, dtype="f32",
                     backward=rng.random() < 0.7, **kinds)
    causal, backward = rng.random() < 0.7, what == "train"
    n = _log_int(rng, 2, 4096 if backward else 8192)
    most = (500_000_000 if backward else 1_500_000_000) * (1 if causal else 0.5) * (64 / d) / (heads * n * n)
    return _attn(None, rng.randint(1, max(1, min(8, int(most)))), heads if most >= 1 else min(heads, max(1, int(most * heads))),
                 kv if most >= 1 else 1, d, n, n, causal=causal, ragged=rng.random() < 0.5, backward=backward, **kinds)


# ---- what is given before a call ----------------------------------------------------------------------------------
def _lengths(case):
    """Keys of each sample: all of them, or between all and half of them."""
    n, batch = case["n_kv"], case["batch"]
    return [n - (b * n) // (2 * batch) if case["ragged"] else n for b in range(batch)]


def _table(buckets, distance, both):
    """The bucket of every distance (key position - query position) from -distance to +distance."""
    rel = torch.arange(-distance, distance + 1, dtype=torch.float64)
    half = buckets // 2 if both else buckets
    away = rel.abs() if both else (-rel).clamp_min(0)
    exact_ones = half // 2
    steps = torch.log(away.clamp_min(1) / exact_ones) / math.log(distance / exact_ones) * (half - exact_ones)
    far = (exact_ones + torch.floor(steps + 1e-9)).clamp_max(half - 1)
    bucket = torch.where(away < exact_ones, away, far)
    return (bucket + (half * (rel > 0) if both else 0)).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    rng = torch.tensor([seed * 1000003 + 17, seed % 1000], dtype=torch.int64, device="cuda")
    if case["kind"] == "drop":
        return dict(case=case, y=normal(case["rows"], case["width"]), x=normal(case["rows"], case["width"]) if case["residual"] else None,
                    rng=rng)
    if case["kind"] == "norm":
        rows, width = case["rows"], case["width"]
        st = dict(case=case, x=normal(rows, width) * 2 + 0.5, y=normal(rows, width), weight=1 + 0.2 * normal(width), bias=0.2 * normal(width), rng=rng)
        if case["backward"]:
            st.update(dn=normal(rows, width), dh=normal(rows, width))
        return st
    B, H, KV, D, nq, nk = (case[k] for k in ("batch", "heads", "kv_heads", "head_dim", "n_q", "n_kv"))
    lengths = _lengths(case)
    st = dict(case=case, q=normal(B, H, nq, D), k=normal(B, KV, nk, D), v=normal(B, KV, nk, D), bias=normal(case["buckets"], H),
              table=_table(case["buckets"], case["distance"], not case["causal"]).cuda(), scale=1 / math.sqrt(D),
              lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda") if case["ragged"] else None,
              start=torch.tensor([n - nq for n in lengths], dtype=torch.int32, device="cuda") if case["at_end"] else None)
    if case["backward"]:
        st["d_o"] = normal(B, H, nq, D)
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return (_run_attn if kind == "attn" else _run_drop if kind == "drop" else _run_norm)(st, st["case"])


def _run_attn(st, case):
    if own:
        import paper_2407_08330_amd as hdt
        args = dict(causal=case["causal"], lengths=st["lengths"], q_start=st["start"])
        o, lse = hdt.hdt_rel_attn_fwd(st["q"], st["k"], st["v"], st["bias"], st["table"], st["scale"], **args)
        if not case["backward"]:
            return {"o": o, "lse": lse}
        dq, dk, dv, dbias = hdt.hdt_rel_attn_bwd(st["q"], st["k"], st["v"], st["bias"], st["table"], o, lse, st["d_o"], st["scale"], **args)
        return {"o": o, "dq": dq, "dk": dk, "dv": dv, "dbias": dbias}
    return _plain_attn(st, case)


def _run_drop(st, case):
    if own:
        import paper_2407_08330_amd as hdt
        return hdt.hdt_dropout_add(st["y"], case["p"], st["rng"], site=3, x=st["x"])
    y = st["y"].float() * _kept(st["y"].numel(), case["p"], st["rng"], 3).view_as(st["y"])
    return (y if st["x"] is None else st["x"].float() + y).to(st["y"].dtype)


def _run_norm(st, case):
    drop = dict(p=case["p"], rng=st["rng"], site=5)
    if own:
        import paper_2407_08330_amd as hdt
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(st["x"], st["weight"], st["bias"], 1e-5, y=st["y"], **drop)
        if not case["backward"]:
            return {"n": n, "h": h}
        dx, dy, dw, db = hdt.hdt_add_norm_bwd(st["dn"], h, st["weight"], mean, rstd, dh=st["dh"], **drop)
        return {"n": n, "h": h, "dx": dx, "dy": dy, "dw": dw, "db": db}
    return _plain_norm(st, case)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _product(a, b):
    """The two halves of the 64-bit products of 32-bit numbers."""
    x = a * b
    return (x >> 32) & 0xFFFFFFFF, x & 0xFFFFFFFF


def _kept(n, p, rng, site):
    """The factor of each of n elements: 0, or 65536 / (65536 - t) with t = p in steps of 1 / 65536.  Eight elements share a block
    of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011), 16 bits each from the lowest on; counter: the block's number, the site,
    the step's two halves; key: the seed's."""
    t = int(p * 65536 + 0.5)
    at = torch.arange((n + 7) // 8, device=rng.device)
    low, high = rng & 0xFFFFFFFF, (rng >> 32) & 0xFFFFFFFF
    c0, c1, c2, c3 = at & 0xFFFFFFFF, torch.full_like(at, site), low[1].expand_as(at), high[1].expand_as(at)
    k0, k1 = low[0], high[0]
    for _ in range(10):
        h0, l0 = _product(c0, 0xD2511F53)
        h1, l1 = _product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)
    u = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(-1)[:n]
    return (u >= t).float() * (65536 / (65536 - t))


def _plain_norm(st, case):
    dtype = st["x"].dtype
    w, b = st["weight"].float(), st["bias"].float()
    kept = _kept(st["x"].numel(), case["p"], st["rng"], 5).view_as(st["x"]) if case["p"] > 0 else torch.ones_like(st["x"], dtype=torch.float32)
    h = st["x"].float() + st["y"].float() * kept
    mean = h.mean(-1, keepdim=True)
    rstd = ((h - mean).square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    hat = (h - mean) * rstd
    n = hat * w + b
    if not case["backward"]:
        return {"n": n.to(dtype), "h": h.to(dtype)}
    dn = st["dn"].float()
    g = dn * w
    dx = st["dh"].float() + rstd * (g - g.mean(-1, keepdim=True) - hat * (g * hat).mean(-1, keepdim=True))
    dw, db = (dn * hat).sum(0, dtype=torch.float64), dn.sum(0, dtype=torch.float64)
    return {"n": n.to(dtype), "h": h.to(dtype), "dx": dx.to(dtype), "dy": (dx * kept).to(dtype), "dw": dw.to(dtype), "db": db.to(dtype)}


def _plain_attn(st, case):
    q, k, v, dtype = st["q"], st["k"], st["v"], st["q"].dtype
    (B, H, nq, D), (KV, nk), M = q.shape, k.shape[1:3], case["distance"]
    G, dev = H // KV, q.device
    lengths = torch.full((1,), nk, device=dev) if st["lengths"] is None else st["lengths"]
    start = torch.zeros((1,), device=dev, dtype=torch.int64) if st["start"] is None else st["start"]
    pos = start.long()[:, None, None] + torch.arange(nq, device=dev)[:, None]      # [.][nq][1]
    key, n = torch.arange(nk, device=dev), lengths.long()[:, None, None]
    rel = key - pos                                                                # [.][nq][nk]
    seen = (key < n) & (pos < n) & (pos >= 0)
    if case["causal"]:
        seen = seen & (rel <= 0)
    seen = seen[:, None, None]
    at = st["table"].long()[rel.clamp(-M, M) + M]
    by_head = st["bias"].float().t().reshape(KV, G, -1)
    qf, kf, vf = q.float().view(B, KV, G, nq, D), k.float()[:, :, None], v.float()[:, :, None]
    s = torch.matmul(qf, kf.transpose(-1, -2)).mul_(st["scale"])
    s = s.add_(by_head[:, :, at].movedim(2, 0)).masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    prob = s.sub_(top).exp_()
    total = prob.sum(-1, keepdim=True)
    lse = (total.log() + top).view(B, H, nq)
    prob = prob.div_(torch.where(total == 0, 1, total))
    o = torch.matmul(prob, vf).view(B, H, nq, D).to(dtype)
    if not case["backward"]:
        return {"o": o, "lse": lse}
    do = st["d_o"].float().view(B, KV, G, nq, D)
    dv = torch.matmul(prob.transpose(-1, -2), torch.where(seen.any(-1, keepdim=True), do, 0)).sum(2)
    ds = torch.matmul(do, vf.transpose(-1, -2))
    ds = ds.sub_((ds * prob).sum(-1, keepdim=True)).mul_(prob)
    del prob
    dq = torch.matmul(ds, kf).mul_(st["scale"]).view(B, H, nq, D)
    dk = torch.matmul(ds.transpose(-1, -2), qf).mul_(st["scale"]).sum(2)
    # the rows one below the other, each shifted by one against the next: a column for each distance
    slid = torch.nn.functional.pad(ds.view(B, H, nq, nk).flip(-2), (0, nq)).view(B, H, -1)[:, :, : nq * (nq + nk - 1)]
    slid = slid.view(B, H, nq, nq + nk - 1).sum(-2, dtype=torch.float64)
    rel = torch.arange(nq + nk - 1, device=dev) - (nq - 1) - start.long()[:, None].expand(B, 1)
    at = st["table"].long()[rel.clamp(-M, M) + M].reshape(-1)
    dbias = torch.zeros(st["bias"].shape, dtype=torch.float64, device=dev).index_add_(0, at, slid.transpose(1, 2).reshape(-1, H))
    return {"o": o, "dq": dq.to(dtype), "dk": dk.to(dtype), "dv": dv.to(dtype), "dbias": dbias.to(dtype)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "drop":
        n = case["rows"] * case["width"]
        return {"bytes": n * size * (3 if case["residual"] else 2), "flops": 2 * n}
    if case["kind"] == "norm":
        n = case["rows"] * case["width"]
        return {"bytes": n * size * (4 + (5 if case["backward"] else 0)), "flops": n * (9 + (15 if case["backward"] else 0))}
    B, H, KV, D, nq, nk = (case[k] for k in ("batch", "heads", "kv_heads", "head_dim", "n_q", "n_kv"))
    pairs = rows = keys = 0
    for n in _lengths(case):
        first = n - nq if case["at_end"] else 0
        real = max(0, min(nq, n - first))
        rows, keys = rows + real, keys + n
        pairs += real * first + real * (real + 1) // 2 if case["causal"] else real * n
    tensors = (4 + 4 if case["backward"] else 2) * H * rows * D + (2 + 2 + 2 if case["backward"] else 2) * KV * keys * D
    return {"bytes": size * tensors + 4 * H * B * nq, "flops": (14 if case["backward"] else 4) * D * H * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(st, case)
    if case["kind"] == "drop":
        y = st["y"].double() * _exact_kept(st["y"].shape, case["p"], st["rng"], 3)
        return y if st["x"] is None else y + st["x"].double()
    x, y, w, b = (st[k].double() for k in ("x", "y", "weight", "bias"))
    factor = _exact_kept(x.shape, case["p"], st["rng"], 5)
    h = x + y * factor
    centred = h - h.sum(1, keepdim=True) / case["width"]
    std = torch.sqrt((centred ** 2).sum(1, keepdim=True) / case["width"] + 1e-5)
    out = {"n": centred / std * w + b, "h": h}
    if case["backward"]:
        dn, dh = st["dn"].double(), st["dh"].double()
        # the derivative of centred / std taken apart: through the centring, and through the deviation
        dc = dn * w / std - centred * ((dn * w * centred).sum(1, keepdim=True) / (case["width"] * std ** 3))
        dx = dh + dc - dc.sum(1, keepdim=True) / case["width"]
        out.update(dx=dx, dy=dx * factor, dw=(dn * centred / std).sum(0), db=dn.sum(0))
    return out


def _exact_kept(shape, p, rng, site):
    """The factors again, the 32-bit products from 16-bit parts, one word of the blocks at a time."""
    n, t, mask = math.prod(shape), round(p * 65536), 0xFFFFFFFF
    if p == 0:
        return torch.ones(shape, dtype=torch.float64, device="cuda")
    seed, step = (int(v) & 0xFFFFFFFFFFFFFFFF for v in rng.tolist())

    def times(a, m):
        low, mid = a * (m & 0xFFFF), a * (m >> 16)
        mid = mid + (low >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    block = torch.arange((n + 7) // 8, device="cuda")
    word = [block, torch.full_like(block, site), torch.full_like(block, step & mask), torch.full_like(block, step >> 32)]
    for i in range(10):
        first, second = (((seed & mask) + i * 0x9E3779B9) & mask), (((seed >> 32) + i * 0xBB67AE85) & mask)
        a, b = times(word[0], 0xD2511F53), times(word[2], 0xCD9E8D57)
        word = [b[0] ^ word[1] ^ first, b[1], a[0] ^ word[3] ^ second, a[1]]
    kept = torch.empty((block.numel(), 8), dtype=torch.float64, device="cuda")
    for i in range(4):
        kept[:, 2 * i] = (word[i] % 65536 >= t).double()
        kept[:, 2 * i + 1] = (word[i] // 65536 >= t).double()
    return kept.reshape(-1)[:n].reshape(shape) / (1 - t / 65536)


def _exact_attn(st, case):
    q, k, v, bias = (st[x].double() for x in ("q", "k", "v", "bias"))
    B, H, nq, D = q.shape
    KV, nk, buckets, distance, dev = case["kv_heads"], case["n_kv"], case["buckets"], case["distance"], q.device
    # the first distance of each bucket of one direction, in whole numbers: bucket e + j begins where (n / e)^L >= (m / e)^j
    half = buckets if case["causal"] else buckets // 2
    e = half // 2
    L = half - e
    first = list(range(e + 1))
    for j in range(1, L):
        n = first[-1]
        while n ** L < e ** (L - j) * distance ** j:
            n += 1
        first.append(n)
    first = torch.tensor(first[1:], device=dev)
    out = {"o": torch.zeros_like(q), "lse": torch.full((B, H, nq), -math.inf, dtype=torch.float64, device=dev)}
    if case["backward"]:
        out.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v), dbias=torch.zeros_like(bias))
    for b, n in enumerate(_lengths(case)):
        begin = n - nq if case["at_end"] else 0
        lo, hi = max(0, -begin), max(0, min(nq, n - begin))  # the rows that stand for positions
        if hi <= lo:
            continue
        away = torch.arange(n, device=dev) - (begin + torch.arange(lo, hi, device=dev))[:, None]
        bucket = torch.bucketize(away.abs(), first, right=True)
        bucket = torch.where(away > 0, 0, bucket) if case["causal"] else torch.where(away > 0, bucket + half, bucket)
        for h in range(H):
            g = h // (H // KV)
            score = (q[b, h, lo:hi] @ k[b, g, :n].t()) * st["scale"] + bias[bucket, h]
            if case["causal"]:
                score[away > 0] = -math.inf
            lse = torch.logsumexp(score, 1)
            prob = torch.exp(score - lse[:, None])
            out["lse"][b, h, lo:hi] = lse
            out["o"][b, h, lo:hi] = prob @ v[b, g, :n]
            if not case["backward"]:
                continue
            do = st["d_o"][b, h, lo:hi].double()
            delta = (do * out["o"][b, h, lo:hi]).sum(1, keepdim=True)
            ds = prob * (do @ v[b, g, :n].t() - delta)
            out["dq"][b, h, lo:hi] = (ds @ k[b, g, :n]) * st["scale"]
            out["dk"][b, g, :n] += (ds.t() @ q[b, h, lo:hi]) * st["scale"]
            out["dv"][b, g, :n] += prob.t() @ do
            for u in range(buckets):
                out["dbias"][u, h] += torch.where(bucket == u, ds, 0).sum()
    if case["backward"]:
        del out["lse"]
    return out
