"""Self-attention with a relative position bias on non-finite values in REAL rows: a NaN reaches every row that sees it, O and LSE, however
the keys are divided among workgroups; rows that cannot see it keep their results.  A score of plus infinity has no softmax and
counts as a NaN does, one of minus infinity is a weight of zero."""
import numpy as np
import pytest

from gpu_common import from_dev, say
from rel_reference import check, half_step
from test_gpu_rel_attn import Problem, dev

pytestmark = pytest.mark.gpu

B, H, KV, D = 2, 4, 2, 64
# name: rows, keys, causal; every way a forward divides its keys: the waves of a workgroup, workgroups whose results are joined, tiles
FORMS = {
    "whole": (200, 200, True), "whole, both ways": (200, 200, False), "several tiles": (520, 520, True), "token": (1, 700, True), "token in pieces": (1, 3000, True),
    "tokens of shared heads in pieces": (7, 3000, True), "chunk": (40, 700, True), "chunk in pieces": (130, 4100, True), "chunk in pieces, both ways": (130, 4100, False),
}
KINDS = {"nan": np.nan, "inf": np.inf, "-inf": -np.inf}


def problem(form, dtype):
    nq, nk, causal = FORMS[form]
    return Problem(B, H, KV, nq, nk, D, dtype=dtype, causal=causal, lengths=[nk, nk - 3], starts=[nk - nq, nk - 3 - nq])


def poisoned(p, tensor, sample, head, row, column, value, dtype):
    """The problem with `value` in a row of q, k or v: in one column, or (None) in all."""
    i = "qkv".index(tensor)
    x = (p.q, p.k, p.v)[i].copy()
    x[sample, head, row, slice(None) if column is None else column] = value
    p.dev = list(p.dev)
    p.dev[i] = dev(x, dtype)
    return x


def scores(p, q, k):
    """A [B][H][nq][nk] of the definition, minus infinity where a key is not visible, and which pairs are visible."""
    nq, nk = q.shape[2], k.shape[2]
    M = (len(p.table) - 1) // 2
    pos = np.asarray(p.starts)[:, None, None] + np.arange(nq)[:, None]
    rel = np.arange(nk) - pos
    n = np.asarray(p.lengths)[:, None, None]
    seen = (np.arange(nk) < n) & (pos >= 0) & (pos < n) & ((rel <= 0) | (not p.causal))
    with np.errstate(all="ignore"):
        # (a sum of products with infinities is a NaN where their signs differ, in any order)
        a = np.stack([[q[b, h] @ k[b, h // (H // KV)].T * p.scale + p.bias[p.table[np.clip(rel[b], -M, M) + M], h] for h in range(H)] for b in range(B)])
    return np.where(seen[:, None], a, -np.inf), np.broadcast_to(seen[:, None], a.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("tensor", ["q", "k", "v"])
def test_forward(form, tensor, dtype):
    import torch
    nq, nk, causal = FORMS[form]
    u = half_step(dtype)
    for kind, value in KINDS.items():
        for column in (None, 3):
            p = problem(form, dtype)
            sample, head, row = 1, 1, (nq // 2 if tensor == "q" else nk // 2 if nq == nk else nk - 20 - nq)
            x = poisoned(p, tensor, sample, head, row, column, value, dtype)
            q, k, v = (x if t == tensor else y for t, y in zip("qkv", (p.q, p.k, p.v)))
            a, seen = scores(p, q, k)
            bad_score = (np.isnan(a) | np.isposinf(a)).any(-1)               # rows whose softmax does not exist
            with np.errstate(all="ignore"):
                top = a.max(-1, keepdims=True)
                w = np.where(seen, np.exp(a - np.where(np.isfinite(top), top, 0)), 0)
                total = w.sum(-1, keepdims=True)
                w = w / np.where(total == 0, 1, total)
                group = np.repeat(v, H // KV, 1)
                o_want, size = w @ np.where(np.isfinite(group), group, 0), w @ np.where(np.isfinite(group), np.abs(group), 0)
                lse_want = np.where(total == 0, -np.inf, np.log(total) + np.where(np.isfinite(top), top, 0))[..., 0]
            # results that a non-finite value of v goes into
            sees_v = seen.astype(np.float32) @ (~np.isfinite(group)).astype(np.float32) > 0
            # rows of the poisoned key's head from which the causal mask hides it and that may share a tile with it: anything
            loose = np.zeros(a.shape[:3], bool)
            if causal and tensor != "q":
                pos = np.asarray(p.starts)[:, None] + np.arange(nq)
                heads = slice(head * (H // KV), (head + 1) * (H // KV))
                loose[sample, heads] = ((pos[sample] < row) & (pos[sample] > row - 192))[None]
            for workspace in (None, torch.empty(16, dtype=torch.uint8, device="cuda")):   # the second: too little for pieces
                o, lse = (from_dev(t).astype(np.float64) for t in p.forward(workspace=workspace))
                tag = f"{form} {tensor} {kind} column {column} {'one piece' if workspace is not None else ''}"
                assert np.isnan(o[bad_score]).all(), f"{tag}: o of a row whose softmax does not exist"
                assert np.isnan(lse[bad_score]).all(), f"{tag}: lse of such a row"
                assert not np.isfinite(o[sees_v]).any(), f"{tag}: o over a non-finite value of v"
                other = ~bad_score & ~loose
                assert np.array_equal(np.isfinite(lse[other]), np.isfinite(lse_want[other])), f"{tag}: lse elsewhere"
                # P and O are rounded, scores have fp32's error (64 products of about 0.1 and their sum: 2e-5) and so has their sum's
                # logarithm, once more in the weights
                fine = other & np.isfinite(lse_want)
                assert np.abs(lse[fine] - lse_want[fine]).max() <= 1e-4, tag
                ok = fine[..., None] & ~sees_v
                off = np.abs(o - o_want) - (u * (size + np.abs(o_want)) * 1.02 + 4e-4)
                assert (off[ok] <= 0).all(), f"{tag}: o elsewhere, {off[ok].max():.3g}"
            if tensor == "q":
                assert bad_score.sum() == 1 and bad_score[sample, head, row]
            elif kind == "nan" and tensor == "k":
                assert bad_score.sum() == seen[sample, head * (H // KV):(head + 1) * (H // KV), :, row].sum() > 0
    say(f"    {form} {tensor} {dtype}: {int(bad_score.sum())} rows without a softmax")


@pytest.mark.parametrize("dtype,width", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("nk", [700, 3000])
def test_a_query_of_nan_is_no_row_without_keys(nk, dtype, width):
    """One token of one sample, all its heads; the other sample's are untouched, bit for bit."""
    import torch
    p = Problem(2, 4, 2, 1, nk, width, dtype=dtype, starts=[nk - 1, nk - 1])
    o, lse = p.forward()
    p.dev[0] = p.dev[0].clone()
    p.dev[0][1] = float("nan")
    o2, lse2 = p.forward()
    assert bool(torch.isnan(o2[1]).all()) and bool(torch.isnan(lse2[1]).all())
    assert torch.equal(o2[0], o[0]) and torch.equal(lse2[0], lse[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tensor", ["q", "k", "v", "d_o"])
def test_backward(tensor, dtype):
    """The gradients that the definition takes a NaN into are NaN, those of other heads' groups and samples are what they are without."""
    n, sample, head, row = 300, 1, 1, 100
    clean = Problem(B, H, KV, n, n, D, dtype=dtype)
    ref = clean.reference()
    p = Problem(B, H, KV, n, n, D, dtype=dtype)
    if tensor == "d_o":
        p.dev_d_o = p.dev_d_o.clone()
        p.dev_d_o[sample, head, row] = float("nan")
    else:
        poisoned(p, tensor, sample, head, row, None, np.nan, dtype)
    o, lse = p.forward()
    dq, dk, dv, dbias = (from_dev(t).astype(np.float64) for t in p.backward(o, lse))
    heads = [head] if tensor in ("q", "d_o") else list(range(head * 2, head * 2 + 2))   # query heads that meet it
    group = heads[0] // 2                                                            # their key head
    rows = [row] if tensor in ("q", "d_o") else list(range(row, n))                  # rows that see it
    for h in heads:
        assert np.isnan(dq[sample, h, rows]).all(), "dq of the rows that see it"
        assert np.isnan(dbias[0, h]), "the bias's gradient at distance 0"
    assert np.isnan(dk[sample, group, :max(rows) + 1]).all(), "dk of every key that such a row sees"
    if tensor != "v":
        assert np.isnan(dv[sample, group, :max(rows) + 1]).all(), "dv of every key that such a row sees"
    keep = [h for h in range(H) if h not in heads]
    check(dq[:, keep], ref.dq[:, keep], ref.dq_bound[:, keep], "dq of other heads")
    check(dq[1 - sample], ref.dq[1 - sample], ref.dq_bound[1 - sample], "dq of the other sample")
    check(dbias[:, keep], ref.dbias[:, keep], ref.dbias_bound[:, keep], "dbias of other heads")
    for name, g in (("dk", dk), ("dv", dv)):
        want, bound = getattr(ref, name), getattr(ref, name + "_bound")
        check(g[:, 1 - group], want[:, 1 - group], bound[:, 1 - group], f"{name} of the other key head")
        check(g[1 - sample], want[1 - sample], bound[1 - sample], f"{name} of the other sample")
