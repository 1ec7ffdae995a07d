"""GPU tests of self-attention with a relative position bias: forward and backward against the 64-bit reference (tests/
rel_reference.py), every output within the bound of its own roundings."""
import numpy as np
import pytest

from gpu_common import GuardedWorkspace, busy, from_dev, say, to_dev_bf16
from paper_2407_08330_amd import inputs
from rel_reference import Reference, check, t5_table

pytestmark = pytest.mark.gpu


def dev(x, dtype):
    import torch
    return to_dev_bf16(x.astype(np.float32)) if dtype == "bf16" else torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def values(rng, shape, dtype):
    x = rng.normal(size=shape).astype(np.float32)
    return (inputs.round_to_bf16(x) if dtype == "bf16" else x).astype(np.float64)


class Problem:
    def __init__(self, B, H, KV, nq, nk, D, *, dtype="bf16", bias_dtype=None, causal=True, lengths=None, starts=None, buckets=32,
                 distance=128, table=None, seed=1, scale=None, poison=False):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.causal, self.lengths, self.starts = dtype, causal, lengths, starts
        self.bias_dtype = bias_dtype or dtype
        self.q, self.d_o = values(rng, (B, H, nq, D), dtype), values(rng, (B, H, nq, D), dtype)
        self.k, self.v = values(rng, (B, KV, nk, D), dtype), values(rng, (B, KV, nk, D), dtype)
        self.bias = values(rng, (buckets, H), self.bias_dtype)
        self.table = t5_table(buckets, distance, not causal) if table is None else np.asarray(table, np.int32)
        self.scale = scale or 1 / np.sqrt(D)
        q, k, v, d_o = (x.copy() for x in (self.q, self.k, self.v, self.d_o))
        if poison:  # what does not stand for a position may hold anything
            for b in range(B):
                n, s = (nk if lengths is None else lengths[b]), (0 if starts is None else starts[b])
                k[b, :, n:], v[b, :, n:] = np.nan, np.inf
                pad = [i for i in range(nq) if not 0 <= s + i < n]
                q[b, :, pad], d_o[b, :, pad] = np.nan, -np.inf
        self.dev = [dev(x, dtype) for x in (q, k, v)] + [dev(self.bias, self.bias_dtype), torch.from_numpy(self.table).cuda()]
        self.dev_d_o = dev(d_o, dtype)
        i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.more = dict(causal=causal, lengths=i32(lengths), q_start=i32(starts))

    def reference(self, backward=True):
        return Reference(self.q, self.k, self.v, self.bias, self.table, self.scale, self.causal, self.lengths, self.starts,
                         self.d_o if backward else None, self.dtype, self.bias_dtype)

    def forward(self, **kw):
        import paper_2407_08330_amd as hdt
        return hdt.hdt_rel_attn_fwd(*self.dev, self.scale, **self.more, **kw)

    def backward(self, o, lse, **kw):
        import paper_2407_08330_amd as hdt
        return hdt.hdt_rel_attn_bwd(*self.dev, o, lse, self.dev_d_o, self.scale, **self.more, **kw)

    def check(self, backward=True):
        import torch
        ref = self.reference(backward)
        nan = float("nan")
        o = torch.full_like(self.dev[0], nan)
        lse = torch.full(self.q.shape[:3], nan, dtype=torch.float32, device="cuda")
        self.forward(o=o, lse=lse)
        worst = [check(from_dev(o).astype(np.float64), ref.o, ref.o_bound, "o"), check(lse.cpu().numpy().astype(np.float64), ref.lse, ref.lse_bound, "lse")]
        if backward:
            outs = dict(dq=torch.full_like(self.dev[0], nan), dk=torch.full_like(self.dev[1], nan), dv=torch.full_like(self.dev[1], nan),
                        dbias=torch.full_like(self.dev[3], nan))
            self.backward(o, lse, **outs)
            for name, t in outs.items():
                worst.append(check(from_dev(t).astype(np.float64), getattr(ref, name), getattr(ref, name + "_bound"), name))
        say("    shares of the bounds: " + " ".join(f"{w:.2f}" for w in worst))


SHAPES = [
    # B, H, KV, n, lengths
    (2, 3, 3, 1, None), (1, 2, 1, 2, None), (2, 4, 2, 33, [33, 17]), (1, 2, 2, 64, None), (2, 2, 2, 127, [127, 64]), (1, 2, 2, 128, None),
    (1, 4, 1, 129, None), (4, 3, 1, 200, [200, 1, 0, 131]), (1, 2, 2, 515, None), (2, 1, 1, 300, [257, 300]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}x{s[3]}")
def test_whole_sequences(shape, dtype, D, causal):
    B, H, KV, n, lengths = shape
    say(f"[rel] {shape} {dtype} d={D} causal={causal}")
    Problem(B, H, KV, n, n, D, dtype=dtype, causal=causal, lengths=lengths, poison=lengths is not None).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("buckets,distance,both", [(32, 128, False), (64, 512, False), (16, 40, True), (2, 1024, False), (4, 1024, True), (4, 2, True)])
def test_buckets(buckets, distance, both, dtype):
    say(f"[rel] buckets {buckets} up to {distance}, both ways {both}, {dtype}")
    Problem(1, 2, 2, 430, 430, 64, dtype=dtype, causal=not both, buckets=buckets, distance=distance).check()


@pytest.mark.parametrize("dtype,bias_dtype", [("bf16", "f32"), ("f32", "bf16")])
def test_bias_of_another_type(dtype, bias_dtype):
    Problem(2, 2, 2, 150, 150, 64, dtype=dtype, bias_dtype=bias_dtype).check()


def test_a_table_of_ones_own():
    """Any bucket at any distance, entries outside the buckets counting as the nearest one inside."""
    rng = np.random.default_rng(9)
    for causal in (True, False):
        Problem(1, 2, 1, 333, 333, 64, causal=causal, buckets=7, table=rng.integers(-3, 11, size=2 * 60 + 1)).check()


CHUNKS = [
    # B, H, KV, nq, nk, lengths
    (3, 4, 2, 1, 300, [300, 1, 0]), (1, 12, 12, 1, 1000, None), (2, 8, 1, 1, 2050, [2050, 1999]), (2, 6, 2, 5, 700, [700, 3]),
    (2, 4, 4, 130, 600, [600, 129]), (1, 12, 1, 20, 400, None), (2, 16, 4, 3, 4100, [4100, 64]), (40, 16, 8, 1, 90, None),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("shape", CHUNKS, ids=lambda s: f"{s[0]}x{s[1]}-{s[2]}x{s[3]}of{s[4]}")
def test_new_tokens_at_the_end_of_a_cache(shape, dtype, D, causal):
    """Lengths shorter than the chunk leave rows in front that stand for nothing."""
    B, H, KV, nq, nk, lengths = shape
    say(f"[rel] {shape} {dtype} d={D} causal={causal}")
    Problem(B, H, KV, nq, nk, D, dtype=dtype, causal=causal, lengths=lengths, starts=[n - nq for n in (lengths or [nk] * B)],
            poison=True).check(backward=B * H * nq * nk < 300_000)


def test_a_token_after_the_other_is_the_whole_sequence():
    """Generating n positions one by one gives the rows of one call over all of them, within the bounds of both."""
    import torch
    import paper_2407_08330_amd as hdt
    n = 70
    p = Problem(2, 4, 2, n, n, 64)
    ref = p.reference(backward=False)
    q, k, v, bias, table = p.dev
    for i in (0, 1, 31, 32, 63, 69):
        lengths = torch.full((2,), i + 1, dtype=torch.int32, device="cuda")
        o, lse = hdt.hdt_rel_attn_fwd(q[:, :, i:i + 1].contiguous(), k, v, bias, table, p.scale, lengths=lengths, q_start=lengths - 1)
        check(from_dev(o).astype(np.float64), ref.o[:, :, i:i + 1], ref.o_bound[:, :, i:i + 1], f"o of token {i}")
        check(lse.cpu().numpy().astype(np.float64), ref.lse[:, :, i:i + 1], ref.lse_bound[:, :, i:i + 1], f"lse of token {i}")


@pytest.mark.parametrize("start", [-2 ** 31, -5000, 5000, 2 ** 31 - 1])
def test_windows_far_outside_the_sequence(start):
    Problem(2, 2, 2, 40, 100, 64, starts=[start, 60], poison=True).check()


@pytest.mark.parametrize("causal", [True, False])
def test_hidden_buckets_and_rows_without_keys(causal):
    """A bias of minus infinity hides a bucket: rows that see nothing else have no result and no gradient."""
    p = Problem(1, 2, 2, 200, 200, 64, causal=causal)
    import torch
    p.bias[0, 0] = -np.inf          # distance 0: row 0 of head 0 sees nothing in the causal form
    p.bias[1:3, 1] = -np.inf
    p.bias[p.table[0], 0] = -np.inf  # all far keys behind
    p.dev[3] = dev(p.bias, "bf16")
    ref = p.reference()
    o, lse = p.forward()
    if causal:
        assert np.isneginf(ref.lse[0, 0, 0])
    check(from_dev(o).astype(np.float64), ref.o, ref.o_bound, "o")
    check(lse.cpu().numpy().astype(np.float64), ref.lse, ref.lse_bound, "lse")
    for name, t in zip(("dq", "dk", "dv", "dbias"), p.backward(o, lse)):
        check(from_dev(t).astype(np.float64), getattr(ref, name), getattr(ref, name + "_bound"), name)
    p.bias[:] = -np.inf
    p.dev[3] = dev(p.bias, "bf16")
    o, lse = p.forward()
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
    assert all(bool((t == 0).all()) for t in p.backward(o, lse))


@pytest.mark.parametrize("low", [float(np.finfo(np.float32).min), -1e9, -1e6])
@pytest.mark.parametrize("scale", [0.125, 1.0, 3.0])
def test_a_bias_of_the_lowest_value(scale, low):
    """Finite values that stand for a mask hide a bucket like minus infinity does; a value short of them is a bias."""
    import torch
    p = Problem(1, 3, 3, 150, 150, 64, scale=scale, bias_dtype="f32")
    p.dev[3][:, 0] = low
    p.dev[3][1:, 1] = low
    p.dev[3][:, 2] += -1e4
    o, lse = p.forward()
    assert bool((o[0, 0] == 0).all()) and bool(torch.isneginf(lse[0, 0]).all())
    assert np.array_equal(from_dev(o)[0, 1], p.v[0, 1].astype(np.float32)), "head 1 sees itself alone"
    assert bool(torch.isfinite(lse[0, 1:]).all())
    dq, dk, dv, dbias = p.backward(o, lse)
    assert all(bool((t[0, 0] == 0).all()) for t in (dq, dk, dv)) and bool((dbias[:, 0] == 0).all())
    assert bool((dbias[1:, 1] == 0).all()) and np.array_equal(from_dev(dv)[0, 1], p.d_o[0, 1].astype(np.float32))
    p.bias[:, :2], p.bias[:, 2] = -np.inf, p.dev[3][:, 2].double().cpu().numpy()
    ref = p.reference()
    check(from_dev(o)[:, 2].astype(np.float64), ref.o[:, 2], ref.o_bound[:, 2], "o")
    check(from_dev(dq)[:, 2].astype(np.float64), ref.dq[:, 2], ref.dq_bound[:, 2], "dq")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Views of a fused projection [batch][rows][3][heads][head_dim], results into views of [batch][rows][heads][head_dim]; the
    same bits as from dense tensors, and nothing written between the rows."""
    import torch
    B, H, n, D = 2, 3, 140, 64
    p = Problem(B, H, H, n, n, D, dtype=dtype, lengths=[140, 77])
    q, k, v, bias, table = p.dev
    o, lse = p.forward()
    grads = p.backward(o, lse)
    fused = torch.full((B, n, 3, H, D + 16), float("nan"), dtype=q.dtype, device="cuda")[..., 8:8 + D]
    for i, t in enumerate((q, k, v)):
        fused[:, :, i] = t.transpose(1, 2)
    p.dev = [fused[:, :, i].transpose(1, 2) for i in range(3)] + [bias, table]
    out = [torch.full((B, n, H, 2 * D), 7.0, dtype=q.dtype, device="cuda") for _ in range(5)]
    view = [t[..., :D].transpose(1, 2) for t in out]
    view[4].copy_(p.dev_d_o)
    p.dev_d_o = view[4]
    o2, lse2 = p.forward(o=view[0])
    grads2 = p.backward(o2, lse2, dq=view[1], dk=view[2], dv=view[3])
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    assert all(torch.equal(a, b) for a, b in zip(grads, grads2))
    assert all(bool((t[..., D:] == 7).all()) for t in out[:4])


def test_broadcast_inputs():
    """One cache for all samples, one query for all heads: gradients are those of the expanded tensors."""
    import torch
    p = Problem(3, 4, 2, 90, 90, 64)
    q, k, v, bias, table = p.dev
    q, k, v = q[:, :1].expand(3, 4, 90, 64), k[:1].expand(3, 2, 90, 64), v[:1, :1].expand(3, 2, 90, 64)
    results = []
    for t in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        p.dev = [*t, bias, table]
        o, lse = p.forward()
        results.append((o, lse, *p.backward(o, lse)))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_the_same_bits_every_time():
    import torch
    p = Problem(2, 4, 2, 700, 700, 64, lengths=[700, 411])
    o, lse = p.forward()
    first = (o, lse, *p.backward(o, lse))
    for _ in range(5):
        o, lse = p.forward()
        assert all(torch.equal(a, b) for a, b in zip(first, (o, lse, *p.backward(o, lse))))


def test_empty_calls():
    import torch
    import paper_2407_08330_amd as hdt
    bias, table = torch.ones(32, 4, device="cuda"), hdt.hdt_rel_table(32, 128)
    for B, nq, nk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        q, k, v = (torch.ones(B, 4, n, 64, device="cuda") for n in (nq, nk, nk))
        o, lse = hdt.hdt_rel_attn_fwd(q, k, v, bias, table, 0.125)
        assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
        grads = hdt.hdt_rel_attn_bwd(q, k, v, bias, table, o, lse, torch.ones_like(q), 0.125,
                                     dk=torch.full_like(k, float("nan")), dbias=torch.full_like(bias, float("nan")))
        assert all(bool((g == 0).all()) for g in grads)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("buckets,distance", [(32, 128), (64, 512), (16, 40), (4, 3), (320, 1024)])
def test_table(buckets, distance, both):
    import paper_2407_08330_amd as hdt
    got = hdt.hdt_rel_table(buckets, distance, both).cpu().numpy()
    assert np.array_equal(got, t5_table(buckets, distance, both))


def test_workspaces_are_not_exceeded_and_not_needed():
    import torch
    import paper_2407_08330_amd as hdt
    from paper_2407_08330_amd import binding
    p = Problem(1, 8, 2, 1, 3000, 64, starts=[2999])
    c = binding._rel_attn_call(*p.dev, p.scale, True, p.more["lengths"], p.more["q_start"])
    lib = hdt.load_library()
    need = lib.hdt_rel_attn_fwd_workspace_bytes(c)
    assert need > 0
    ws = GuardedWorkspace(need)
    o, lse = p.forward(workspace=ws.view)
    ws.check()
    o2, lse2 = p.forward(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))  # too little: the keys stay together
    ref = p.reference(backward=False)
    for a, l in ((o, lse), (o2, lse2)):
        check(from_dev(a).astype(np.float64), ref.o, ref.o_bound, "o")
        check(l.cpu().numpy().astype(np.float64), ref.lse, ref.lse_bound, "lse")
    p = Problem(2, 4, 2, 333, 333, 128)
    o, lse = p.forward()
    ws = GuardedWorkspace(lib.hdt_rel_attn_bwd_workspace_bytes(binding._rel_attn_call(*p.dev, p.scale, True, None, None)))
    p.backward(o, lse, workspace=ws.view)
    ws.check()


def test_on_another_stream():
    import torch
    p = Problem(2, 4, 2, 257, 257, 64)
    o, lse = p.forward()
    want = (o, lse, *p.backward(o, lse))
    side = torch.cuda.Stream()
    busy()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    o2, lse2 = p.forward(stream=side)          # behind the side stream's work, not the current stream's
    got = (o2, lse2, *p.backward(o2, lse2, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_and_replayed():
    """A forward and backward in a graph: new values in the same tensors at every replay, lengths among them, with eager calls between;
    a second graph shares the workspace."""
    import torch
    import paper_2407_08330_amd as hdt
    from paper_2407_08330_amd import binding
    B, H, n, D = 2, 4, 300, 64
    p = Problem(B, H, 2, n, n, D, lengths=[300, 150])
    q, k, v, bias, table = p.dev
    lib = hdt.load_library()
    c = binding._rel_attn_call(*p.dev, p.scale, True, p.more["lengths"], None)
    ws = torch.empty(max(lib.hdt_rel_attn_fwd_workspace_bytes(c), lib.hdt_rel_attn_bwd_workspace_bytes(c), 1 << 20), dtype=torch.uint8, device="cuda")
    o, lse = p.forward()
    outs = [torch.empty_like(t) for t in (o, lse, q, k, v, bias)]
    token = dict(q=q[:, :, :1].contiguous(), lengths=torch.tensor([290, 31], dtype=torch.int32, device="cuda"))
    token["start"] = token["lengths"] - 1
    t_out = [torch.empty_like(token["q"]), torch.empty(B, H, 1, dtype=torch.float32, device="cuda")]

    def step():
        p.forward(o=outs[0], lse=outs[1], workspace=ws)
        p.backward(outs[0], outs[1], dq=outs[2], dk=outs[3], dv=outs[4], dbias=outs[5], workspace=ws)

    def one():
        hdt.hdt_rel_attn_fwd(token["q"], k, v, bias, table, p.scale, lengths=token["lengths"], q_start=token["start"], o=t_out[0], lse=t_out[1], workspace=ws)

    step(), one()
    torch.cuda.synchronize()
    graphs = []
    for f in (step, one):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    for r in range(4):
        for t in (q, k, v, bias, p.dev_d_o, token["q"]):
            t.copy_(torch.randn_like(t))
        p.more["lengths"].copy_(torch.tensor([300 - 60 * r, 1 + 90 * r], dtype=torch.int32))
        for t in (*outs, *t_out):
            t.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*outs, *t_out)]
        step(), one()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*outs, *t_out))), f"replay {r}"


def test_a_cache_beyond_32_bit_offsets():
    """A batch whose key tensor is larger than 4 GiB: the last sample's results are those of a small call on a copy of it."""
    import torch
    import paper_2407_08330_amd as hdt
    B, H, n, D = 36, 4, 131072, 128     # 4.8 GB a tensor
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.empty(B, H, n, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for t in (k, v):
        for b in (0, B - 1):
            t[b] = torch.randn(H, n, D, generator=gen, device="cuda").bfloat16()
    q = torch.randn(B, H, 1, D, generator=gen, device="cuda").bfloat16()
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    lengths[0], lengths[-1] = 5, n
    bias, table = torch.randn(32, H, generator=gen, device="cuda"), hdt.hdt_rel_table(32, 128)
    o, lse = hdt.hdt_rel_attn_fwd(q, k, v, bias, table, 0.1, lengths=lengths, q_start=lengths - 1)
    a = (q[-1].double() @ k[-1].double().transpose(-1, -2)) * 0.1
    far = n - 1 - torch.arange(n, device="cuda").clamp(max=n - 1)
    a += bias.double()[table.long()[(-far).clamp(-128, 128) + 128]].t()[:, None]
    want = torch.softmax(a, -1) @ v[-1].double()
    # P and O are rounded to bf16, scores of a few units in fp32
    most = 2.0 ** -8 * (torch.softmax(a, -1) @ v[-1].double().abs() + want.abs()) * 1.02 + 1e-6
    assert bool(((o[-1].double() - want).abs() <= most).all())
    assert float((lse[-1].double() - torch.logsumexp(a, -1)).abs().max()) <= 1e-5 * 20
    assert bool((o[1:-1] == 0).all()) and bool(torch.isneginf(lse[1:-1]).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("B,H,KV", [(10, 6, 3), (11, 10, 10), (25, 7, 7)])
def test_many_heads(B, H, KV, dtype, D, causal):
    """60, 110 and 175 heads of 140 rows: the tile shapes that calls take as their heads become many (tiles of 32, 64 and 128 rows in the
    forward, 64 and 128 in the backward)."""
    say(f"[rel] {B} x {H}/{KV} heads x 140 {dtype} d={D} causal={causal}")
    lengths = [140 - 9 * b % 141 for b in range(B)]
    Problem(B, H, KV, 140, 140, D, dtype=dtype, causal=causal, lengths=lengths, distance=20, poison=True).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("B,H,KV,nq,nk,lengths", [(2, 2, 2, 100, 2200, [2200, 700]), (1, 3, 3, 40, 2100, None), (2, 4, 2, 150, 2049, [2049, 149]),
                                                  (1, 1, 1, 2100, 2100, None), (1, 30, 1, 9, 2500, None)])
def test_pieces_of_the_keys(B, H, KV, nq, nk, lengths, dtype, D, causal):
    """Many keys, few rows or heads: the keys divided among workgroups, some of which may have none, in every tile shape that does so."""
    say(f"[rel] {B} x {H}/{KV} heads x {nq} of {nk} {dtype} d={D} causal={causal}")
    Problem(B, H, KV, nq, nk, D, dtype=dtype, causal=causal, lengths=lengths, starts=[n - nq for n in (lengths or [nk] * B)], poison=True).check(backward=nq < 200)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("H,nq,distance", [(16, 1, 128), (16, 1, 127), (17, 1, 128), (16, 9, 128), (2, 1, 1024), (2, 140, 1024)])
def test_tables_that_fill_the_lds(H, nq, distance, dtype, D, causal):
    """Query heads of one key head, each with its bias by distance in LDS beside the rings: up to the last bytes there are, and beyond."""
    say(f"[rel] {H}/1 heads x {nq} of 300, distances up to {distance}, {dtype} d={D} causal={causal}")
    Problem(2, H, 1, nq, 300, D, dtype=dtype, causal=causal, lengths=[300, 150], starts=[300 - nq, 150 - nq], distance=distance, poison=True).check()
