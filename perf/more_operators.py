"""The rest of a layer around the hierarchical attention: embeddings, the gated feed-forward block, the norms around a block.

  embed  token embeddings: rows of a table by ids, scaled; forward, or forward and the table's gradient
  ffn    gated feed-forward block: two projections, activation, product, third projection; forward, or forward and backward
  gnorm  the norm behind a block, its gate, the scaled residual and the norm in front of the next block in one; forward, or forward and backward

Every operator stands here in its plain form too (elementary torch operations in 32 bits), and `exact` says what the definition
gives in 64 bits.  `own` selects between the plain forms and the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases --------------------------------------------------------------------------------------------------
def _embed(name, tokens, vocab, width, *, backward, dtype="bf16", table="bf16", scale=1.0, pads=False):
    """dtype: of the embeddings; table: of the table and its gradient; pads: some ids are -1."""
    case = dict(kind="embed", tokens=tokens, vocab=vocab, width=width, backward=backward, dtype=dtype, table=table, scale=scale, pads=pads)
    return dict(case, name=name) if name else case


def _ffn(name, rows, width, inner, act, *, backward, dtype="bf16"):
    case = dict(kind="ffn", rows=rows, width=width, inner=inner, act=act, backward=backward, dtype=dtype)
    return dict(case, name=name) if name else case


def _gnorm(name, rows, width, *, backward, rms=True, gate=True, bias=False, scale=1.0, dtype="bf16"):
    case = dict(kind="gnorm", rows=rows, width=width, backward=backward, rms=rms, gate=gate, bias=bias, scale=scale, dtype=dtype)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one new token of each of four documents, where latency counts
        _embed("embed-tokens-4", 4, 32768, 768, backward=False, scale=math.sqrt(768)),
        # a padded batch of prompts, the table kept in 32 bits
        _embed("embed-prompts-16384", 16384, 32768, 768, backward=False, table="f32", scale=math.sqrt(768), pads=True),
        # a training step on 4 x 8192 positions: words as frequent as words are
        _embed("embed-train-32768", 32768, 32768, 768, backward=True, scale=math.sqrt(768)),
        # a small vocabulary in 32 bits (operators and digits of nested lists), rows that are no multiple of eight
        _embed("embed-train-f32-5003", 5003, 101, 513, backward=True, dtype="f32", table="f32", pads=True),
        # one new token of one document in a decoder layer, where latency counts
        _ffn("ffn-token-1", 1, 768, 2048, "gelu_tanh", backward=False),
        # a full serving batch, one new token each
        _ffn("ffn-tokens-32", 32, 1024, 2816, "silu", backward=False),
        # a prompt of 8192 positions through a layer, forward only
        _ffn("ffn-prompt-8192", 8192, 768, 2048, "gelu_tanh", backward=False),
        # the block in a training step on 4 x 8192 positions
        _ffn("ffn-train-32768", 32768, 768, 2048, "gelu_tanh", backward=True),
        # a short ragged batch, sizes that no tile divides
        _ffn("ffn-train-1999", 1999, 1000, 2504, "gelu", backward=True),
        # the path that checks a model's numbers
        _ffn("ffn-check-f32-512", 512, 384, 1000, "silu", backward=True, dtype="f32"),
        # four new tokens between two blocks
        _gnorm("gnorm-tokens-4", 4, 768, backward=False),
        # between two blocks of a training step on 4 x 8192 positions
        _gnorm("gnorm-train-32768", 32768, 768, backward=True, rms=False, bias=True, scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["embed", "embed", "embed", "tokens", "prompt", "train", "train", "check", "gnorm", "gnorm", "gnorm"])
    if what in ("embed", "gnorm"):
        width = rng.choice([rng.randint(16, 1500), rng.choice([512, 768, 1024, 2048])])
        backward = rng.random() < 0.6
        if what == "embed":
            dtype, table = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
            return _embed(None, _log_int(rng, 1, max(1, 25_000_000 // width)), _log_int(rng, 16, max(16, 25_000_000 // width)), width, backward=backward,
                          dtype=dtype, table=table, scale=rng.choice([1.0, math.sqrt(width)]), pads=rng.random() < 0.4)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _gnorm(None, _log_int(rng, 1, max(1, (25_000_000 if dtype == "bf16" else 10_000_000) // width)), width, backward=backward, rms=rng.random() < 0.5,
                      gate=rng.random() < 0.7, bias=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 1.7]), dtype=dtype)
    width = rng.choice([256, 512, 768, 1024, 1536, 8 * rng.randint(8, 192), rng.randint(64, 1536)])
    inner = max(64, int(width * rng.uniform(2.0, 4.0)) // 8 * 8) if rng.random() < 0.85 else rng.randint(64, 4 * width)
    act = rng.choice(["silu", "gelu", "gelu_tanh"])
    if what == "tokens":
        return _ffn(None, _log_int(rng, 1, 200), width, inner, act, backward=False)
    if what == "check":
        return _ffn(None, _log_int(rng, 1, min(2048, 1_000_000_000 // (width * inner))), width, inner, act, backward=rng.random() < 0.7, dtype="f32")
    if what == "prompt":
        return _ffn(None, _log_int(rng, 64, min(32768, 50_000_000_000 // (width * inner))), width, inner, act, backward=False)
    return _ffn(None, _log_int(rng, 16, min(32768, 25_000_000_000 // (width * inner))), width, inner, act, backward=True)


# ---- what is given before a call ----------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, times=1.0, plus=0.0, dtype=dtype):
        return (torch.randn(shape, generator=gen, device="cuda") * times + plus).to(dtype)

    if case["kind"] == "embed":
        tokens, vocab, width, table = case["tokens"], case["vocab"], case["width"], DTYPES[case["table"]]
        # id r is met about 1 / (r + 1) as often as id 0, as the words of a vocabulary that was made by frequency
        u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
        ids = torch.exp(u * math.log(vocab + 1)).long().sub(1).clamp(0, vocab - 1).to(torch.int32)
        if case["pads"]:
            ids[torch.rand(tokens, generator=gen, device="cuda") < 0.1] = -1
        st = dict(case=case, ids=ids, table=normal(vocab, width, times=1 / math.sqrt(width), dtype=table))
        if case["backward"]:
            st["dx"] = normal(tokens, width)
        return st
    rows, width = case["rows"], case["width"]
    if case["kind"] == "ffn":
        inner = case["inner"]
        st = dict(case=case, x=normal(rows, width), w_gate=normal(inner, width, times=1 / math.sqrt(width)), w_up=normal(inner, width, times=1 / math.sqrt(width)),
                  w_down=normal(width, inner, times=1 / math.sqrt(inner)))
        if case["backward"]:
            st["dy"] = normal(rows, width)
        return st
    st = dict(case=case, x=normal(rows, width, times=2.0, plus=0.5), y=normal(rows, width, times=0.7), post_weight=normal(width, times=0.2, plus=1.0),
              weight=normal(width, times=0.2, plus=1.0), gate=normal(width, times=0.3, plus=0.5) if case["gate"] else None,
              post_bias=normal(width, times=0.2) if case["bias"] else None, bias=normal(width, times=0.2) if case["bias"] else None)
    if case["backward"]:
        st.update(dn=normal(rows, width), dh=normal(rows, width))
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    return (_run_embed if kind == "embed" else _run_ffn if kind == "ffn" else _run_gnorm)(st, st["case"])


def _run_embed(st, case):
    dtype, table = DTYPES[case["dtype"]], st["table"]
    if own:
        import paper_2407_08330_amd as hdt
        x = hdt.hdt_embed_fwd(st["ids"], table, case["scale"], dtype=dtype)
        if not case["backward"]:
            return {"x": x}
        return {"x": x, "dtable": hdt.hdt_embed_bwd(st["dx"], st["ids"], case["vocab"], case["scale"], dtype=table.dtype)}
    real = (st["ids"] >= 0)[:, None]
    at = st["ids"].long().clamp_min(0)
    x = torch.where(real, table[at].float() * case["scale"], 0).to(dtype)
    if not case["backward"]:
        return {"x": x}
    dx = torch.where(real, st["dx"].double() * case["scale"], 0)
    return {"x": x, "dtable": torch.zeros(table.shape, dtype=torch.float64, device=x.device).index_add_(0, at, dx).to(table.dtype)}


def _run_ffn(st, case):
    if own:
        import paper_2407_08330_amd as hdt
        weights = st["w_gate"], st["w_up"], st["w_down"]
        y, *kept = hdt.hdt_ffn_fwd(st["x"], *weights, case["act"], train=case["backward"])
        if not case["backward"]:
            return {"y": y}
        dx, dwg, dwu, dwd = hdt.hdt_ffn_bwd(st["dy"], st["x"], *weights, *kept)
        return {"y": y, "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    return _plain_ffn(st, case)


def _run_gnorm(st, case):
    if own:
        import paper_2407_08330_amd as hdt
        n, h, stats = hdt.hdt_gate_norm_fwd(st["x"], st["y"], st["post_weight"], st["weight"], gate=st["gate"], post_bias=st["post_bias"], bias=st["bias"],
                                            scale=case["scale"], eps=1e-5, rms=case["rms"])
        if not case["backward"]:
            return {"n": n, "h": h}
        dx, dy, dpw, dw, dg, dpb, db = hdt.hdt_gate_norm_bwd(st["dn"], h, st["y"], stats, st["post_weight"], st["weight"], gate=st["gate"], post_bias=st["post_bias"],
                                                             bias=case["bias"], dh=st["dh"], scale=case["scale"], rms=case["rms"])
        out = {"n": n, "h": h, "dx": dx, "dy": dy, "dpost_weight": dpw, "dweight": dw, "dgate": dg, "dpost_bias": dpb, "dbias": db}
        return {k: v for k, v in out.items() if v is not None}
    return _plain_gnorm(st, case)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_ffn(st, case):
    dtype = st["x"].dtype
    x, wg, wu, wd = (st[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(g, case["act"])
    h = a * u
    y = (h @ wd.t()).to(dtype)
    if not case["backward"]:
        return {"y": y}
    dy = st["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    return {"y": y, "dx": (dg @ wg + du @ wu).to(dtype), "dw_gate": (dg.t() @ x).to(dtype), "dw_up": (du.t() @ x).to(dtype), "dw_down": (dy.t() @ h).to(dtype)}


def _centre(t, rms):
    return 0 if rms else t.mean(-1, keepdim=True)


def _plain_gnorm(st, case):
    dtype, rms = st["x"].dtype, case["rms"]
    x, y, wp, w = (st[k].float() for k in ("x", "y", "post_weight", "weight"))
    gate = 1 if st["gate"] is None else st["gate"].float()
    cy = y - _centre(y, rms)
    ry = (cy.square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    yhat = cy * ry
    c = yhat * wp + (st["post_bias"].float() if case["bias"] else 0)
    h = case["scale"] * x + gate * c
    ch = h - _centre(h, rms)
    rh = (ch.square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    hhat = ch * rh
    n = hhat * w + (st["bias"].float() if case["bias"] else 0)
    out = {"n": n.to(dtype), "h": h.to(dtype)}
    if not case["backward"]:
        return out
    dn = st["dn"].float()
    g = dn * w
    dh = st["dh"].float() + rh * (g - _centre(g, rms) - hhat * (g * hhat).mean(-1, keepdim=True))
    dc = dh * gate
    g = dc * wp
    dy = ry * (g - _centre(g, rms) - yhat * (g * yhat).mean(-1, keepdim=True))

    def column(t):
        return t.sum(0, dtype=torch.float64).to(dtype)

    out.update(dx=(case["scale"] * dh).to(dtype), dy=dy.to(dtype), dpost_weight=column(dc * yhat), dweight=column(dn * hhat))
    if case["gate"]:
        out["dgate"] = column(dh * c)
    if case["bias"]:
        out.update(dpost_bias=column(dc), dbias=column(dn))
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "embed":
        elements, table = case["tokens"] * case["width"], 2 if case["table"] == "bf16" else 4
        # rows of the table that a pass meets, about: those of ids that come at least once
        per = math.log(case["vocab"] + 1)
        met = sum(-math.expm1(-case["tokens"] * math.log1p(1 / r) / per) * n for r, n in _ranks(case["vocab"]))
        read = min(met, case["tokens"]) * case["width"] * table
        if not case["backward"]:
            return {"bytes": int(read + elements * size + 4 * case["tokens"]), "flops": elements}
        return {"bytes": int(read + 2 * elements * size + 4 * case["tokens"] + case["vocab"] * case["width"] * table), "flops": 3 * elements}
    rows, width = case["rows"], case["width"]
    if case["kind"] == "ffn":
        weights, product = 3 * width * case["inner"], 2 * rows * width * case["inner"]
        if not case["backward"]:
            return {"bytes": size * (2 * rows * width + weights), "flops": 3 * product}
        return {"bytes": size * (4 * rows * width + 2 * weights), "flops": 9 * product}
    n = rows * width
    return {"bytes": n * size * (4 + (4 if case["backward"] else 0)) + 8 * width * size, "flops": n * (14 + (30 if case["backward"] else 0))}


def _ranks(vocab):
    """(a rank, how many ranks it stands for)"""
    r = 1
    while r <= vocab:
        n = min(max(1, r // 16), vocab - r + 1)
        yield r + (n - 1) / 2, n
        r += n


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return (_exact_embed if case["kind"] == "embed" else _exact_ffn if case["kind"] == "ffn" else _exact_gnorm)(st, case)


def _exact_embed(st, case):
    ids = st["ids"].long()
    at = torch.nonzero(ids >= 0)[:, 0]
    x = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
    x[at] = st["table"].double()[ids[at]] * case["scale"]
    if not case["backward"]:
        return {"x": x}
    dtable = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    dtable.index_put_((ids[at],), st["dx"].double()[at], accumulate=True)
    return {"x": x, "dtable": dtable * case["scale"]}


def _exact_ffn(st, case):
    """The definition in 64 bits; torch differentiates it."""
    names = ("x", "w_gate", "w_up", "w_down")
    x, wg, wu, wd = (st[k].double().requires_grad_(case["backward"]) for k in names)
    g = x @ wg.t()
    if case["act"] == "silu":
        a = g / (1 + torch.exp(-g))
    elif case["act"] == "gelu":
        a = g * torch.special.erfc(-g / math.sqrt(2)) / 2
    else:
        a = g / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    y = (a * (x @ wu.t())) @ wd.t()
    if not case["backward"]:
        return {"y": y}
    grads = torch.autograd.grad(y, (x, wg, wu, wd), st["dy"].double())
    return {"y": y.detach(), **dict(zip(("dx", "dw_gate", "dw_up", "dw_down"), grads))}


def _exact_gnorm(st, case):
    """The definition in 64 bits; torch differentiates it."""
    names = [k for k in ("x", "y", "post_weight", "weight", "gate", "post_bias", "bias") if st[k] is not None]
    t = {k: st[k].double().requires_grad_(case["backward"]) for k in names}

    def norm(v, w, b):
        if not case["rms"]:
            v = v - v.sum(1, keepdim=True) / case["width"]
        v = w * v / torch.sqrt((v * v).sum(1, keepdim=True) / case["width"] + 1e-5)
        return v if b is None else v + b

    c = norm(t["y"], t["post_weight"], t.get("post_bias"))
    h = case["scale"] * t["x"] + (c if st["gate"] is None else t["gate"] * c)
    n = norm(h, t["weight"], t.get("bias"))
    if not case["backward"]:
        return {"n": n, "h": h}
    grads = torch.autograd.grad((n, h), [t[k] for k in names], (st["dn"].double(), st["dh"].double()))
    by = {"d" + k: g for k, g in zip(names, grads)}
    return {"n": n.detach(), "h": h.detach(), **{k: by[k] for k in ("dx", "dy", "dpost_weight", "dweight", "dgate", "dpost_bias", "dbias") if k in by}}
