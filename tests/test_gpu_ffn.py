"""GPU tests of the gated feed-forward block against the 64-bit reference (tests/layer_reference.py), each output within the bound of its own
roundings."""
import numpy as np
import pytest

import layer_reference as lr
from gpu_common import GuardedWorkspace, busy, from_dev, say
from rel_reference import check, half_step
from test_gpu_rel_attn import dev, values

pytestmark = pytest.mark.gpu

ACTS = ["silu", "gelu", "gelu_tanh"]


def host(t):
    return from_dev(t).astype(np.float64)


def problem(rows, width, inner, dtype, seed=0):
    rng = np.random.default_rng(rows * 1000 + width + inner + seed)
    x, dy = values(rng, (rows, width), dtype), values(rng, (rows, width), dtype)
    rounded = lambda a: host(dev(a, dtype)) if dtype == "f32" else values_of(a)  # noqa: E731
    wg, wu = (rounded(values(rng, (inner, width), dtype) * 1.5 / np.sqrt(width)) for _ in range(2))
    wd = rounded(values(rng, (width, inner), dtype) / np.sqrt(inner))
    return x, dy, wg, wu, wd


def values_of(a):
    from paper_2407_08330_amd import inputs
    return inputs.round_to_bf16(a.astype(np.float32)).astype(np.float64)


def guarded(shape, dtype):
    """a tensor with 64 elements behind it that stay 7"""
    import torch
    n = int(np.prod(shape))
    room = torch.full((n + 64,), 7.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    return room[:n].view(shape), lambda: bool((room[n:] == 7).all())


def check_call(rows, width, inner, act, dtype):
    import torch
    import paper_2407_08330_amd as hdt
    say(f"[ffn] {rows} x {width} x {inner} {act} {dtype}")
    u = half_step(dtype)
    x, dy, wg, wu, wd = problem(rows, width, inner, dtype)
    xd, *weights = (dev(t, dtype) for t in (x, wg, wu, wd))
    results = {k: guarded((rows, width if k == "y" else inner), dtype) for k in ("y", "by_gate", "by_up", "hidden")}
    ws = GuardedWorkspace(hdt.load_library().hdt_ffn_fwd_workspace_bytes(rows, width, inner, 1, 0 if dtype == "bf16" else 1))
    y, *kept = hdt.hdt_ffn_fwd(xd, *weights, act, **{k: t for k, (t, _) in results.items()}, workspace=ws.view)
    ws.check()
    assert all(ok() for _, ok in results.values())
    want = lr.ffn_inner(x, wg, wu, act, u)
    for name, t in zip(("by_gate", "by_up", "hidden"), kept):
        check(host(t), *want[name], name)
    check(host(y), *lr.ffn_out(host(kept[2]), wd, u), "y")
    ws = GuardedWorkspace(hdt.load_library().hdt_ffn_fwd_workspace_bytes(rows, width, inner, 0, 0 if dtype == "bf16" else 1))
    only = hdt.hdt_ffn_fwd(xd, *weights, act, train=False, workspace=ws.view)
    ws.check()
    assert torch.equal(only[0], y) and only[1:] == (None, None, None)

    grads = {k: guarded(t.shape, dtype) for k, t in zip(("dx", "dw_gate", "dw_up", "dw_down"), (xd, *weights))}
    ws = GuardedWorkspace(hdt.load_library().hdt_ffn_bwd_workspace_bytes(rows, width, inner, 0 if dtype == "bf16" else 1))
    ws.buf[:ws.nbytes] = 0xFF
    got = hdt.hdt_ffn_bwd(dev(dy, dtype), xd, *weights, *kept, **{k: t for k, (t, _) in grads.items()}, workspace=ws.view)
    ws.check()
    assert all(ok() for _, ok in grads.values())
    want = lr.ffn_grads(dy, x, wg, wu, wd, *(host(t) for t in kept), u)
    for name, t in zip(("dx", "dw_gate", "dw_up", "dw_down"), got):
        check(host(t), *want[name], name)


# rows, width, inner: the smallest, sizes on both sides of every tile's border, sizes that are no multiple of eight
SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 128), (2, 768, 256), (3, 7, 5), (5, 24, 40), (16, 64, 64), (17, 72, 200), (31, 33, 65), (32, 128, 384), (33, 136, 264), (64, 256, 512), (65, 64, 72),
         (100, 200, 120), (127, 63, 129), (128, 128, 128), (129, 320, 136), (200, 512, 1032), (255, 256, 256), (256, 264, 520), (257, 520, 264), (300, 100, 1000), (520, 192, 200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,inner", SIZES)
def test_ffn(rows, width, inner, dtype):
    check_call(rows, width, inner, ACTS[(rows + width + inner) % 3], dtype)


# rows on both sides of every number of rows a workgroup, with few columns and with more than a workgroup a compute unit of them; beyond 64, 128 and 192
@pytest.mark.parametrize("rows,width,inner", [(8, 2064, 72), (15, 2049, 65), (16, 2100, 130), (48, 2056, 264), (49, 1032, 2056), (80, 520, 136), (96, 2056, 136), (100, 100, 2060),
                                              (128, 264, 520), (129, 136, 1040), (144, 1111, 77), (177, 88, 2200), (192, 70, 200), (193, 72, 200), (40, 4104, 2056), (64, 4160, 72)])
def test_few_rows(rows, width, inner):
    check_call(rows, width, inner, "gelu", "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,width,inner", [(4, 96, 160), (70, 96, 160), (300, 256, 512)])
def test_activations(rows, width, inner, act, dtype):
    check_call(rows, width, inner, act, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_whole_range(act, dtype):
    """G is set one by one: x is one value, Wg the points, Wu ones."""
    import torch
    import paper_2407_08330_amd as hdt
    points = np.concatenate([np.linspace(-40, 40, 801), [0.0, -0.0, 1e-30, -1e-30, 1e-6, 88.0, -88.0, 1e4, -1e4, 1e19, -1e19, 1e30, -1e30]])
    wg = host(dev(points[:, None], dtype)) if dtype == "f32" else values_of(points[:, None])
    n = len(wg)
    one = np.ones((1, 1))
    t = [dev(v, dtype) for v in (one, wg, np.ones((n, 1)), np.ones((1, n)))]
    y, *kept = hdt.hdt_ffn_fwd(*t, act)
    u = half_step(dtype)
    with np.errstate(over="ignore", invalid="ignore"):
        want = lr.ffn_inner(one, np.clip(wg, -60, 60), np.ones((n, 1)), act, u)
    big = np.abs(wg[:, 0]) > 60
    for name, k in zip(("by_gate", "by_up", "hidden"), kept):
        got, (v, e) = host(k)[0], want[name]
        check(got[~big], v[0][~big], e[0][~big], name)
        far = np.maximum(wg[big, 0], 0) if name != "by_gate" else (wg[big, 0] > 0).astype(float)
        assert np.all(np.abs(got[big] - far) <= 2 * u * np.abs(far) + 1e-6), name


@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_up_to_the_types_largest_values(act, dtype, rows):
    """G is set one by one, as above, up to the largest values of the type, in one row (few rows) and in 300 (tiles).  Out there the activation is g or 0 and
    its slope 1 or 0: the value itself, rounded once, behind factors of 1 that are off by a few 2^-24.  Below -88 the sigmoid is 2^-126 at most (its
    exponential may overflow, or its value be flushed to 0), and 0 below -89: with g, under 89 2^-126."""
    import torch
    import paper_2407_08330_amd as hdt
    most = {"bf16": 2.0 ** 127 * (2 - 2.0 ** -7), "f32": 2.0 ** 127 * (2 - 2.0 ** -23)}[dtype]
    sizes = [88.0, 89.0, 90.0, 100.0, 104.0, 128.0, 200.0, 1e3, 1e10, 1e20, 1e30, 1e33, 1e36, 1e37, 1e38, 3e38, most]
    points = np.array([s * v for v in sizes for s in (1, -1)])
    wg = host(dev(points[:, None], dtype)) if dtype == "f32" else values_of(points[:, None])
    assert abs(wg[-1, 0]) == most
    n, u = len(wg), half_step(dtype)
    t = [dev(v, dtype) for v in (np.ones((rows, 1)), wg, np.ones((n, 1)), np.ones((1, n)))]
    kept = hdt.hdt_ffn_fwd(*t, act)[1:]
    g = wg[:, 0]
    for name, k in zip(("by_gate", "by_up", "hidden"), kept):
        want = (g > 0).astype(float) if name == "by_gate" else np.maximum(g, 0)
        assert np.all(np.abs(host(k) - want) <= (u + 4 * lr.F32) * np.abs(want) + 89 * 2.0 ** -126), (name, g[np.argmax(np.abs(host(k) - want).max(0))])
    # a NaN stays one
    wg[:] = np.nan
    t[1] = dev(wg, dtype)
    assert all(bool(k.isnan().all()) for k in hdt.hdt_ffn_fwd(*t, act)[1:])


@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_infinite_g_gives_what_the_formula_gives(act, dtype, rows):
    import torch
    import paper_2407_08330_amd as hdt
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, wg = torch.ones(rows, 1, device="cuda", dtype=t), torch.tensor([[float("inf")], [-float("inf")], [1.0]], device="cuda", dtype=t)
    _, by_gate, by_up, hidden = hdt.hdt_ffn_fwd(x, wg, torch.ones_like(wg), torch.ones(1, 3, device="cuda", dtype=t), act)
    for k in (by_up, hidden):
        assert bool((k[:, 0] == float("inf")).all()) and bool(k[:, 1].isnan().all())
    assert bool(by_gate[:, :2].isnan().all()) and all(bool(k[:, 2].isfinite().all()) for k in (by_gate, by_up, hidden))


def test_shapes_and_no_rows():
    import torch
    import paper_2407_08330_amd as hdt
    x = torch.randn(2, 3, 16, device="cuda").bfloat16()
    w = [torch.randn(s, device="cuda").bfloat16() for s in ((24, 16), (24, 16), (16, 24))]
    y, *kept = hdt.hdt_ffn_fwd(x, *w)
    assert y.shape == x.shape and all(k.shape == (2, 3, 24) for k in kept)
    flat, *fk = hdt.hdt_ffn_fwd(x.view(6, 16), *w)
    assert torch.equal(flat.view(x.shape), y)
    assert all(torch.equal(a.view(-1), b.view(-1)) for a, b in zip(hdt.hdt_ffn_bwd(y, x, *w, *kept), hdt.hdt_ffn_bwd(flat, x.view(6, 16), *w, *fk)))
    assert hdt.hdt_ffn_fwd(x[0, 0], *w, train=False)[0].shape == (16,)
    for dtype in (torch.bfloat16, torch.float32):
        e, we = torch.empty(0, 16, device="cuda", dtype=dtype), [t.to(dtype) for t in w]
        y, *kept = hdt.hdt_ffn_fwd(e, *we)
        grads = hdt.hdt_ffn_bwd(y, e, *we, *kept, **{k: torch.full_like(t, float("nan")) for k, t in zip(("dw_gate", "dw_up", "dw_down"), we)})
        assert y.shape == (0, 16) and grads[0].shape == (0, 16) and all(bool((g == 0).all()) for g in grads[1:])


@pytest.mark.parametrize("rows,width,inner", [(20, 64, 72), (150, 80, 2056), (300, 256, 264), (300, 60, 100)])
def test_rows_do_not_meet(rows, width, inner):
    """A row's y and dx depend on that row alone: NaN and infinities in others change nothing, whatever tile they share."""
    import torch
    import paper_2407_08330_amd as hdt
    for dtype in ("bf16", "f32"):
        x, dy, *w = problem(rows, width, inner, dtype)
        w = [dev(t, dtype) for t in w]
        outs = []
        for bad in (False, True):
            a, b = x.copy(), dy.copy()
            if bad:
                a[3], b[3], a[rows - 2, 0], b[rows - 2] = np.nan, np.nan, np.inf, -np.inf
            y, *kept = hdt.hdt_ffn_fwd(dev(a, dtype), *w)
            outs.append((y, hdt.hdt_ffn_bwd(dev(b, dtype), dev(a, dtype), *w, *kept)[0]))
        good = [r for r in range(rows) if r not in (3, rows - 2)]
        assert all(torch.equal(p[good], q[good]) for p, q in zip(*outs))
        assert bool(outs[1][0][3].isnan().all()) and bool(outs[1][1][3].isnan().all())


def test_weights_as_rows_of_one_tensor():
    """w_gate and w_up as halves of one projection."""
    import torch
    import paper_2407_08330_amd as hdt
    x, dy, wg, wu, wd = problem(150, 64, 128, "bf16")
    both = torch.cat([dev(wg, "bf16"), dev(wu, "bf16")])
    want = hdt.hdt_ffn_fwd(dev(x, "bf16"), dev(wg, "bf16"), dev(wu, "bf16"), dev(wd, "bf16"))
    got = hdt.hdt_ffn_fwd(dev(x, "bf16"), both[:128], both[128:], dev(wd, "bf16"))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("rows,width,inner", [(3, 64, 128), (700, 256, 512), (1500, 136, 200)])
def test_the_same_bits_every_time_captured_and_on_another_stream(rows, width, inner):
    import torch
    import paper_2407_08330_amd as hdt
    x, dy, *w = (dev(t, "bf16") for t in problem(rows, width, inner, "bf16"))
    lib = hdt.load_library()
    ws = torch.empty(max(16, lib.hdt_ffn_fwd_workspace_bytes(rows, width, inner, 1, 0), lib.hdt_ffn_bwd_workspace_bytes(rows, width, inner, 0)), dtype=torch.uint8, device="cuda")

    def step(**kw):
        y, *kept = hdt.hdt_ffn_fwd(x, *w, "gelu_tanh", **kw)
        return (y, *kept, *hdt.hdt_ffn_bwd(dy, x, *w, *kept, **kw))

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(want, step(workspace=ws)))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):  # two graphs that share a workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(workspace=ws))
        graphs.append(graph)
    for r in range(3):
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(float("nan"))
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, out)), f"replay {r}"
            step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    got = step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_train_step_of_many_rows():
    """Beyond the sizes the reference goes to: the sums over rows against products in 64 bits on the device."""
    import torch
    import paper_2407_08330_amd as hdt
    rows, width, inner = 9001, 520, 1096
    x, dy, *w = (dev(t, "bf16") for t in problem(rows, width, inner, "bf16"))
    y, *kept = hdt.hdt_ffn_fwd(x, *w, "gelu")
    dx, dwg, dwu, dwd = hdt.hdt_ffn_bwd(dy, x, *w, *kept)
    g, up = x.double() @ w[0].double().t(), x.double() @ w[1].double().t()
    cdf = 0.5 * torch.special.erfc(-g / 2 ** 0.5)
    pg, pu = up * (cdf + g * torch.exp(-g * g / 2) / (2 * np.pi) ** 0.5), g * cdf
    dh = dy.double() @ w[2].double()
    dg, du = dh * pg, dh * pu
    want = {"y": (pu * up) @ w[2].double().t(), "dx": dg @ w[0].double() + du @ w[1].double(), "dw_gate": dg.t() @ x.double(), "dw_up": du.t() @ x.double(),
            "dw_down": dy.double().t() @ (pu * up)}
    for name, t in (("y", y), ("dx", dx), ("dw_gate", dwg), ("dw_up", dwu), ("dw_down", dwd)):
        # three roundings of half a step at most in front of a sum of values of both signs, and the result's own: four of a root mean square of at most 2^-8 / sqrt(3)
        off = float((t.double() - want[name]).norm() / want[name].norm())
        assert off <= 2 ** -8 / 3 ** 0.5 * 4 ** 0.5, (name, off)


def test_offsets_beyond_32_bits():
    """Hidden rows behind 2^32 elements: the last rows against a call on them alone (width 64: sums of one order, so the same bits), gradients against
    those of the rows that are not zero."""
    import torch
    import paper_2407_08330_amd as hdt
    rows, width, inner, last = 300_000, 64, 16384, 128
    x, dy, *w = (dev(t, "bf16") for t in problem(last, width, inner, "bf16"))
    big, dbig = (torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    big[-last:], dbig[-last:] = x, dy
    y, *kept = hdt.hdt_ffn_fwd(big, *w)
    want, *few = hdt.hdt_ffn_fwd(x, *w)
    assert all(torch.equal(a[-last:], b) and not bool(a[:-last].any()) for a, b in zip(kept, few))
    # y and the gradients: sums of up to 16384 (or 128) terms in 32 bits, in pieces that the sizes decide: within a step of bf16 and 2^-24 times their number
    def near(a, b):
        off = (a.double() - b.double()).norm() / b.double().norm()
        return float(off) <= 2 ** -8
    assert near(y[-last:], want) and not bool(y[:-last].any())
    got = hdt.hdt_ffn_bwd(dbig, big, *w, *kept)
    ref = hdt.hdt_ffn_bwd(dy, x, *w, *few)
    assert near(got[0][-last:], ref[0]) and not bool(got[0][:-last].any())
    assert all(near(a, b) for a, b in zip(got[1:], ref[1:]))
