"""GPU tests of embedding lookup and the table's gradient against the 64-bit reference (tests/layer_reference.py)."""
import numpy as np
import pytest

import layer_reference as lr
from gpu_common import GuardedWorkspace, busy, from_dev, say
from rel_reference import check, half_step
from test_gpu_rel_attn import dev, values

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")]  # of the table, of the embeddings


def torch_type(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def host(t):
    return from_dev(t).astype(np.float64)


def i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def word_ids(rng, n, vocab, kind):
    if kind == "words":  # the first ids are met most
        return np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1).clip(0)
    if kind == "same":
        return np.full(n, vocab - 1)
    if kind == "none":
        return np.where(rng.random(n) < 0.5, -1, vocab)
    if kind == "runs":  # rows of exactly 32, 64 and one more or less tokens: where blocks of tokens begin and end
        return np.repeat(np.arange(n) % vocab, np.resize([32, 31, 33, 64, 1, 65, 96], n))[:n]
    ids = rng.integers(-2, vocab + 2, n)
    ids[:3] = [2 ** 31 - 1, -2 ** 31, vocab][:min(3, n)]
    return ids


CASES = [(1, 1, 1, "words"), (1, 5, 8, "words"), (2, 300, 7, "any"), (31, 2, 9, "same"), (32, 3, 24, "same"), (33, 3, 24, "same"), (64, 1, 520, "same"), (100, 1000, 513, "any"),
         (1025, 7, 16, "words"), (1000, 600, 768, "words"), (777, 257, 1000, "any"), (300, 50, 40, "none"), (2000, 40, 8, "runs"), (4099, 131, 72, "words"), (5000, 3, 33, "words"),
         (70, 140000, 8, "words")]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("tokens,vocab,width,kind", CASES)
def test_embed(tokens, vocab, width, kind, types):
    import torch
    import paper_2407_08330_amd as hdt
    say(f"[embed] {tokens} of {vocab} x {width} {kind} {types}")
    tt, dt = types
    rng = np.random.default_rng(tokens + width)
    ids = word_ids(rng, tokens, vocab, kind)
    table, d_out, scale = values(rng, (vocab, width), tt), values(rng, (tokens, width), dt), 1.7
    scale32 = float(np.float32(scale))
    room = torch.full((tokens * width + 64,), 7.0, dtype=torch_type(dt), device="cuda")
    out = room[:tokens * width].view(tokens, width)
    assert hdt.hdt_embed_fwd(i32(ids), dev(table, tt), scale, out=out) is out
    check(host(out), *lr.embed(ids, table, scale32, half_step(dt)), "out")
    assert bool((room[tokens * width:] == 7).all())

    poisoned = d_out.copy()
    poisoned[(ids < 0) | (ids >= vocab)] = np.nan  # rows that no row of the table gave
    ws = GuardedWorkspace(hdt.load_library().hdt_embed_bwd_workspace_bytes(tokens, width))
    ws.buf[:ws.nbytes] = 0xFF
    room = torch.full((vocab * width + 64,), 7.0, dtype=torch_type(tt), device="cuda")
    grad = room[:vocab * width].view(vocab, width)
    assert hdt.hdt_embed_bwd(dev(poisoned, dt), i32(ids), vocab, scale, grad=grad, workspace=ws.view) is grad
    ws.check()
    check(host(grad), *lr.embed_grad(d_out, ids, vocab, scale32, half_step(tt)), "grad")
    assert bool((room[vocab * width:] == 7).all())
    again = hdt.hdt_embed_bwd(dev(poisoned, dt), i32(ids), vocab, scale, dtype=torch_type(tt))
    assert torch.equal(again, grad)

    old = values(rng, (vocab, width), tt)
    before = dev(old, tt)
    after = hdt.hdt_embed_bwd(dev(poisoned, dt), i32(ids), vocab, scale, grad=before.clone(), accumulate=True)
    check(host(after), *lr.embed_grad(d_out, ids, vocab, scale32, half_step(tt), old), "accumulated")
    met = np.zeros(vocab, bool)
    met[ids[(ids >= 0) & (ids < vocab)]] = True
    assert torch.equal(after[torch.from_numpy(~met).cuda()], before[torch.from_numpy(~met).cuda()])


def test_shapes_no_tokens_and_rows_without_one():
    import torch
    import paper_2407_08330_amd as hdt
    table = torch.randn(50, 12, device="cuda")
    ids = torch.randint(-1, 50, (2, 3, 5), dtype=torch.int32, device="cuda")
    out = hdt.hdt_embed_fwd(ids, table, dtype=torch.bfloat16)
    assert out.shape == (2, 3, 5, 12) and out.dtype == torch.bfloat16
    grad = hdt.hdt_embed_bwd(out, ids, 50)
    assert grad.shape == (50, 12) and grad.dtype == torch.bfloat16
    assert torch.equal(grad, hdt.hdt_embed_bwd(out.view(30, 12), ids.view(30), 50))
    one = torch.tensor(7, dtype=torch.int32, device="cuda")
    assert torch.equal(hdt.hdt_embed_fwd(one, table), table[7])
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert hdt.hdt_embed_fwd(none, table).shape == (0, 12)
    nan = torch.full((50, 12), float("nan"), device="cuda")
    assert bool((hdt.hdt_embed_bwd(torch.empty(0, 12, device="cuda"), none, 50, grad=nan.clone()) == 0).all())
    assert bool(hdt.hdt_embed_bwd(torch.empty(0, 12, device="cuda"), none, 50, grad=nan, accumulate=True).isnan().all())


@pytest.mark.parametrize("offset", [0, 1, 16])
def test_no_tokens_and_a_workspace_of_no_bytes(offset):
    """Without tokens no workspace is needed: memory behind the address of one of no bytes, aligned or not, is not the call's."""
    import torch
    import paper_2407_08330_amd as hdt
    lib = hdt.load_library()
    assert lib.hdt_embed_bwd_workspace_bytes(0, 12) == 0
    for dtype, code in ((torch.bfloat16, 0), (torch.float32, 1)):
        room = torch.full((4096,), 0x5A, dtype=torch.uint8, device="cuda")
        grad = torch.full((50, 12), float("nan"), dtype=dtype, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        assert lib.hdt_embed_bwd(None, None, 0, 50, 12, 1.0, 0, grad.data_ptr(), code, code, room.data_ptr() + offset, 0, st) == 0
        assert bool((grad == 0).all()) and bool((room == 0x5A).all())
        none = torch.empty(0, dtype=torch.int32, device="cuda")
        grad.fill_(float("nan"))
        hdt.hdt_embed_bwd(torch.empty(0, 12, dtype=dtype, device="cuda"), none, 50, grad=grad, workspace=room[offset:offset + 3])
        assert bool((grad == 0).all()) and bool((room == 0x5A).all())


def test_non_finite_values_stay_in_their_rows():
    import torch
    import paper_2407_08330_amd as hdt
    ids = torch.tensor([3, 1, 3, 2], dtype=torch.int32, device="cuda")
    table = torch.ones(5, 24, device="cuda")
    table[1], table[4] = float("nan"), float("inf")
    out = hdt.hdt_embed_fwd(ids, table)
    assert bool(out[1].isnan().all()) and bool((out[[0, 2, 3]] == 1).all())
    d = torch.ones(4, 24, device="cuda")
    d[0, 3], d[3, 4] = float("nan"), float("inf")
    grad = hdt.hdt_embed_bwd(d, ids, 5)
    assert bool(grad[3, 3].isnan()) and float(grad[2, 4]) == float("inf") and int((~grad.isfinite()).sum()) == 2


@pytest.mark.parametrize("tokens,vocab,width", [(20000, 30000, 768), (40000, 300, 64), (100000, 5, 16)])
def test_large(tokens, vocab, width):
    """Whole numbers in fp32: sums are exact in any order."""
    import torch
    import paper_2407_08330_amd as hdt
    rng = np.random.default_rng(1)
    ids = i32(word_ids(rng, tokens, vocab, "words"))
    d = torch.randint(-3, 4, (tokens, width), device="cuda").float()
    want = torch.zeros(vocab, width, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), d.double())
    assert torch.equal(hdt.hdt_embed_bwd(d, ids, vocab, 2.0).double(), want * 2)
    assert torch.equal(hdt.hdt_embed_bwd(d, ids, vocab, 2.0, grad=torch.ones(vocab, width, device="cuda"), accumulate=True).double(), want * 2 + 1)


@pytest.mark.parametrize("tokens", [4000, 32700, 70001])
def test_many_rows_of_one_share(tokens):
    """All ids are congruent modulo 256: a workgroup of the sort has them all, up to 512 rows, and each wave places up to 256 of them a step, one behind the
    other, whose places the steps before have moved on.  Whole numbers: sums are exact in any order; rows that come once show every single token."""
    import torch
    import paper_2407_08330_amd as hdt
    vocab, width = 131072, 8
    rng = np.random.default_rng(tokens)
    for rows in (2, 100, 512):
        ids = i32(rng.integers(0, rows, tokens) * 256 + 7)
        d = torch.randint(-3, 4, (tokens, width), device="cuda").float()
        want = torch.zeros(vocab, width, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), d.double())
        assert torch.equal(hdt.hdt_embed_bwd(d, ids, vocab).double(), want), rows
    ids = i32(rng.permutation(512) * 256 + 255)
    d = torch.randn(512, width, device="cuda")
    assert torch.equal(hdt.hdt_embed_bwd(d, ids, vocab)[ids.long()], d)


@pytest.mark.parametrize("tokens", [255, 257, 4095, 4096, 4097, 32767, 32768, 32769])
def test_ids_that_begin_anywhere(tokens):
    """Ids at every 4-byte offset, behind them ones that are not theirs; whole numbers: sums are exact in any order."""
    import torch
    import paper_2407_08330_amd as hdt
    vocab, width = 777, 8
    rng = np.random.default_rng(tokens)
    ids = i32(word_ids(rng, tokens, vocab, "any"))
    d = torch.randint(-3, 4, (tokens, width), device="cuda").float()
    real = (ids >= 0) & (ids < vocab)
    want = torch.zeros(vocab, width, device="cuda", dtype=torch.float64).index_add_(0, ids[real].long(), d[real].double())
    for offset in range(4):
        room = torch.full((tokens + 8,), 5, dtype=torch.int32, device="cuda")
        here = room[offset:offset + tokens]
        here.copy_(ids)
        assert torch.equal(hdt.hdt_embed_bwd(d, here, vocab).double(), want)


def test_offsets_beyond_32_bits():
    """A table and a gradient of more than 2^32 elements."""
    import torch
    import paper_2407_08330_amd as hdt
    vocab, width = 140_000, 32768
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    table[vocab - 1], table[vocab - 2] = 3, 5
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab], dtype=torch.int32, device="cuda")
    out = hdt.hdt_embed_fwd(ids, table)
    assert [float(v) for v in out.float().amin(1)] == [3, 0, 5, 0] == [float(v) for v in out.float().amax(1)]
    hdt.hdt_embed_bwd(out, ids, vocab, grad=table)
    assert float(table[vocab - 1].float().amin()) == 3 and float(table[vocab - 2].float().amin()) == 5 and int((table[:vocab - 2] != 0).any()) == 0


def test_captured_and_on_another_stream():
    """Ids that change between replays; two graphs that share a workspace."""
    import torch
    import paper_2407_08330_amd as hdt
    rng = np.random.default_rng(5)
    tokens, vocab, width = 700, 90, 100
    ids = [i32(word_ids(rng, tokens, vocab, k)) for k in ("words", "any", "same", "runs")]
    table, d = torch.randn(vocab, width, device="cuda"), torch.randn(tokens, width, device="cuda")
    ws = torch.empty(hdt.load_library().hdt_embed_bwd_workspace_bytes(tokens, width), dtype=torch.uint8, device="cuda")
    here, out, grads = ids[0].clone(), torch.empty(tokens, width, device="cuda"), [torch.empty(vocab, width, device="cuda") for _ in range(2)]
    hdt.hdt_embed_bwd(d, here, vocab, grad=grads[0], workspace=ws)
    torch.cuda.synchronize()
    graphs = []
    for g in grads:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hdt.hdt_embed_fwd(here, table, 2.0, out=out)
            hdt.hdt_embed_bwd(d, here, vocab, 2.0, grad=g, workspace=ws)
        graphs.append(graph)
    for i in ids:
        here.copy_(i)
        for g, graph in zip(grads, graphs):
            g.fill_(float("nan")), out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(g, hdt.hdt_embed_bwd(d, i, vocab, 2.0)) and torch.equal(out, hdt.hdt_embed_fwd(i, table, 2.0))
    want = hdt.hdt_embed_fwd(ids[0], table), hdt.hdt_embed_bwd(d, ids[0], vocab)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    got = hdt.hdt_embed_fwd(ids[0], table, stream=side), hdt.hdt_embed_bwd(d, ids[0], vocab, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
