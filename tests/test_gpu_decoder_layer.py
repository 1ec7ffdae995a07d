"""The operators around the attention in a row, as a decoder's layer calls them: dropout of the embeddings, norm, self-attention with a
relative position bias, residual + dropout + norm, dropout + residual; a training step with its gradients, the same step captured and
replayed, and token after token behind a cache."""
import numpy as np
import pytest

import norm_reference
import rel_reference

pytestmark = pytest.mark.gpu

HEADS, KV, D, WIDTH = 4, 2, 64, 96
SCALE, P, EPS = 0.11, 0.2, 1e-5
LENGTHS = [77, 41]


class Layer:
    """The layer on the device; weights in ``dtype``."""

    def __init__(self, dtype, seed=3, n=77):
        import torch
        import paper_2407_08330_amd as hdt
        self.hdt, self.torch, self.dtype, self.n, self.B = hdt, torch, dtype, n, len(LENGTHS)
        g = torch.Generator().manual_seed(seed)
        make = lambda *s, by=1.0: (by * torch.randn(s, generator=g, dtype=torch.float64)).to(dtype).cuda()  # noqa: E731
        self.e, self.d_out = make(self.B, n, WIDTH), make(self.B, n, WIDTH)
        self.w_qkv, self.w_o, self.w_f = make(WIDTH, (HEADS + 2 * KV) * D, by=0.1), make(HEADS * D, WIDTH, by=0.06), make(WIDTH, WIDTH, by=0.1)
        self.bias = make(32, HEADS)
        self.norms = [(1 + make(WIDTH, by=0.2), make(WIDTH, by=0.2)) for _ in range(2)]
        self.rng = torch.tensor([11, 5], dtype=torch.int64, device="cuda")
        self.table = hdt.hdt_rel_table(32, 128)
        self.lengths = torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()

    def split(self, qkv):
        """views [B][heads][n][D] of [B][n][heads * D], as the projection leaves them"""
        x = qkv.unflatten(-1, (-1, D)).transpose(1, 2)
        return x[:, :HEADS], x[:, HEADS:HEADS + KV], x[:, HEADS + KV:]

    def heads_last(self, n):
        flat = self.torch.empty(self.B, n, HEADS * D, dtype=self.dtype, device="cuda")
        return flat, flat.unflatten(-1, (HEADS, D)).transpose(1, 2)

    def step(self):
        """out and the gradients of everything"""
        t, hdt, drop = self.torch, self.hdt, dict(p=P, rng=self.rng)
        (w1, b1), (w2, b2) = self.norms
        x = hdt.hdt_dropout_add(self.e, P, self.rng, 0)
        n1, h1, mean1, rstd1 = hdt.hdt_add_norm_fwd(x, w1, b1, EPS)
        qkv = n1 @ self.w_qkv
        q, k, v = self.split(qkv)
        o_flat, o = self.heads_last(self.n)
        _, lse = hdt.hdt_rel_attn_fwd(q, k, v, self.bias, self.table, SCALE, lengths=self.lengths, o=o)
        y = o_flat @ self.w_o
        n2, h2, mean2, rstd2 = hdt.hdt_add_norm_fwd(h1, w2, b2, EPS, y=y, site=1, **drop)
        z = n2 @ self.w_f
        out = hdt.hdt_dropout_add(z, P, self.rng, 2, x=h2)

        dz = hdt.hdt_dropout_add(self.d_out, P, self.rng, 2)
        dn2 = dz @ self.w_f.T
        dx2, dy, dw2, db2 = hdt.hdt_add_norm_bwd(dn2, h2, w2, mean2, rstd2, dh=self.d_out, site=1, **drop)
        d_flat = dy @ self.w_o.T
        d_o = d_flat.unflatten(-1, (HEADS, D)).transpose(1, 2)
        d_qkv = t.empty_like(qkv)
        dq, dk, dv = self.split(d_qkv)
        _, _, _, dbias = hdt.hdt_rel_attn_bwd(q, k, v, self.bias, self.table, o, lse, d_o, SCALE, lengths=self.lengths, dq=dq, dk=dk, dv=dv)
        dn1 = d_qkv @ self.w_qkv.T
        dx1, _, dw1, db1 = hdt.hdt_add_norm_bwd(dn1, h1, w1, mean1, rstd1, dh=dx2)
        de = hdt.hdt_dropout_add(dx1, P, self.rng, 0)
        flat = lambda a: a.reshape(-1, a.shape[-1])  # noqa: E731
        return dict(out=out, e=de, bias=dbias, w1=dw1, b1=db1, w2=dw2, b2=db2, w_qkv=flat(n1).T @ flat(d_qkv), w_o=flat(o_flat).T @ flat(dy),
                    w_f=flat(n2).T @ flat(dz))

    def reference(self):
        """The same in 64 bits, by torch's differentiation of the formulas."""
        torch = self.torch
        names = dict(e=self.e, bias=self.bias, w1=self.norms[0][0], b1=self.norms[0][1], w2=self.norms[1][0], b2=self.norms[1][1], w_qkv=self.w_qkv,
                     w_o=self.w_o, w_f=self.w_f)
        w = {name: a.detach().cpu().double().requires_grad_() for name, a in names.items()}
        seed, step = self.rng.tolist()
        f = [torch.from_numpy(norm_reference.factors(self.e.numel(), P, seed, step, site)).view(self.e.shape) for site in range(3)]
        norm = lambda h, a, b: (h - h.mean(-1, keepdim=True)) / (h.var(-1, unbiased=False, keepdim=True) + EPS).sqrt() * a + b  # noqa: E731
        h1 = w["e"] * f[0]
        q, k, v = self.split(norm(h1, w["w1"], w["b1"]) @ w["w_qkv"])
        i = torch.arange(self.n)
        distance = i[None, :] - i[:, None]
        bucket = torch.from_numpy(rel_reference.t5_table(32, 128, False)).long()[distance.clamp(-128, 128) + 128]
        group = lambda a: a.repeat_interleave(HEADS // KV, dim=1)  # noqa: E731
        s = q @ group(k).transpose(-1, -2) * SCALE + w["bias"][bucket].permute(2, 0, 1)
        length = torch.tensor(LENGTHS)[:, None, None, None]
        s = s.masked_fill((distance > 0) | (i >= length), float("-inf"))
        o = (s.softmax(-1) @ group(v)) * (i[:, None] < length)
        h2 = h1 + (o.transpose(1, 2).flatten(2) @ w["w_o"]) * f[1]
        out = h2 + (norm(h2, w["w2"], w["b2"]) @ w["w_f"]) * f[2]
        out.backward(self.d_out.cpu().double())
        return dict(out=out.detach(), **{name: a.grad for name, a in w.items()})


def test_training_step_against_64_bits():
    """fp32.  Every result passes through at most 4 products of 96 or 256 terms, 4 norms of 96, 3 sums over 64 columns and 3 over 77 keys,
    and one over 154 rows: under 2000 terms, each rounded to 2^-24 of the sum of magnitudes; norms, softmax and cancellation inside
    these sums raise that by less than 8."""
    import torch
    layer = Layer(torch.float32)
    want, got = layer.reference(), layer.step()
    for name, x in got.items():
        off = (x.cpu().double() - want[name]).norm() / want[name].norm()
        print(f"[layer] {name} {off:.2e}", flush=True)
        assert off < 8 * 2000 * 2.0 ** -24, name


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_captured_step_is_the_eager_one(name):
    """Replays with the generator's step raised between them, against eager calls at those steps, bit for bit."""
    import torch
    layer = Layer({"bf16": torch.bfloat16, "f32": torch.float32}[name])
    eager = []
    for _ in range(3):
        eager.append({k: x.clone() for k, x in layer.step().items()})
        layer.rng[1] += 1
    layer.rng[1] -= 3
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer.step()
    for i, want in enumerate(eager):
        graph.replay()
        torch.cuda.synchronize()
        for k, x in held.items():
            assert torch.equal(x, want[k]), (i, k)
        layer.rng[1] += 1
    assert not torch.equal(eager[0]["out"], eager[1]["out"])


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_tokens_behind_a_cache_are_the_rows_of_the_whole(name):
    """Queries one at a time (and the first of them as one chunk), over a cache with room behind its last key, give the whole sequence's
    rows: both are within the forward's bound of the same value, and so within two bounds of each other."""
    import torch
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[name]
    layer = Layer(dtype)
    hdt, n, room = layer.hdt, layer.n, layer.n + 23
    qkv = layer.e @ layer.w_qkv
    q, k, v = layer.split(qkv)
    whole, lse = hdt.hdt_rel_attn_fwd(q, k, v, layer.bias, layer.table, SCALE)
    r = rel_reference.Reference(*(x.cpu().double().numpy() for x in (q, k, v, layer.bias)), rel_reference.t5_table(32, 128, False), SCALE, True, dtype=name)
    rel_reference.check(whole.cpu().double().numpy(), r.o, r.o_bound, "whole")
    cache_k, cache_v = (torch.full((layer.B, KV, room, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    first = n - 6
    got = torch.zeros_like(whole)
    for at, rows in [(0, first)] + [(i, 1) for i in range(first, n)]:
        cache_k[:, :, at:at + rows], cache_v[:, :, at:at + rows] = k[:, :, at:at + rows], v[:, :, at:at + rows]
        start = torch.full((layer.B,), at, dtype=torch.int32, device="cuda")
        o, l = hdt.hdt_rel_attn_fwd(q[:, :, at:at + rows], cache_k, cache_v, layer.bias, layer.table, SCALE, lengths=start + rows, q_start=start)
        got[:, :, at:at + rows] = o
        assert np.all(np.abs((l - lse[:, :, at:at + rows]).cpu().numpy()) <= 2 * r.lse_bound[:, :, at:at + rows])
    rel_reference.check(got.cpu().double().numpy(), r.o, r.o_bound, "tokens")
