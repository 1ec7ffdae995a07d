"""GPU tests of the norms around a block against the 64-bit reference (tests/layer_reference.py), each output within the bound of its own
roundings."""
import numpy as np
import pytest

import layer_reference as lr
from gpu_common import GuardedWorkspace, busy, from_dev, say
from rel_reference import check, half_step
from test_gpu_norm import as_type
from test_gpu_rel_attn import dev, values

pytestmark = pytest.mark.gpu

ROWS = [(1, 1), (1, 768), (4, 768), (5, 7), (9, 9), (130, 1000), (7, 511), (6, 513), (300, 64), (2, 1024), (3, 1025), (5, 2048), (2, 2049), (3, 4096), (2, 4097), (2, 8192),
        (2, 8193), (2, 32768), (2, 32761), (4100, 24)]
GRADS = ("dx", "dy", "dpost_weight", "dweight", "dgate", "dpost_bias", "dbias")


def host(t):
    return from_dev(t).astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", ROWS)
def test_gate_norm(rows, width, dtype):
    import torch
    import paper_2407_08330_amd as hdt
    say(f"[gate_norm] {rows} x {width} {dtype}")
    rng = np.random.default_rng(rows * 40000 + width)
    u = half_step(dtype)
    for rms, with_gate, with_bias, with_dh, wdt, scale in ((True, True, False, True, dtype, 1.0), (False, True, True, True, "f32", 0.5), (False, False, True, False, "bf16", -1.25),
                                                           (True, False, False, False, dtype, 1.0)):
        x, y, dn, dh = (values(rng, (rows, width), dtype) for _ in range(4))
        y = as_type(y * 0.7 + 0.25, dtype).astype(np.float64)
        wp, w, gate, bp, b = (as_type(values(rng, (width,), wdt) / 4 + m, wdt).astype(np.float64) for m in (1, 1, 0.5, 0, 0))
        v = dict(post_weight=wp, weight=w, gate=gate if with_gate else None, post_bias=bp if with_bias else None, bias=b if with_bias else None)
        d = {k: None if t is None else dev(t, wdt) for k, t in v.items()}
        n, h, stats = hdt.hdt_gate_norm_fwd(dev(x, dtype), dev(y, dtype), **d, scale=scale, eps=1e-3, rms=rms)
        full = [np.full(width, c) if t is None else t for t, c in ((v["post_bias"], 0.0), (v["gate"], 1.0), (v["bias"], 0.0))]
        want = lr.gate_norm(x, y, wp, full[0], full[1], w, full[2], scale, float(np.float32(1e-3)), rms, u)
        for name, t in (("h", h), ("n", n), ("stats", stats)):
            check(host(t), *want[name], name)
        if rms:
            assert bool((stats[[0, 2]] == 0).all())
        ws = GuardedWorkspace(hdt.load_library().hdt_gate_norm_bwd_workspace_bytes(rows, width))
        got = hdt.hdt_gate_norm_bwd(dev(dn, dtype), h, dev(y, dtype), stats, d["post_weight"], d["weight"], gate=d["gate"], post_bias=d["post_bias"], bias=with_bias,
                                    dh=dev(dh, dtype) if with_dh else None, scale=scale, rms=rms, workspace=ws.view)
        ws.check()
        want = lr.gate_norm_grads(dn, dh if with_dh else 0 * dh, host(h), y, host(stats), wp, full[0], full[1], w, scale, rms, u, half_step(wdt))
        assert [t is not None for t in got[4:]] == [with_gate, with_bias, with_bias]
        for name, t in zip(GRADS, got):
            if t is not None:
                check(host(t), *want[name], f"{name} rms={rms}")


def test_against_add_norm():
    """With a post norm that changes nothing it is the residual and its norm."""
    import torch
    import paper_2407_08330_amd as hdt
    x, y = torch.randn(50, 768, device="cuda"), torch.randn(50, 768, device="cuda")
    y = (y - y.mean(1, keepdim=True)) / y.std(1, keepdim=True, unbiased=False)
    one, w, b = torch.ones(768, device="cuda"), torch.randn(768, device="cuda"), torch.randn(768, device="cuda")
    n, h, _ = hdt.hdt_gate_norm_fwd(x, y, one, w, bias=b, eps=0.0)
    want, wh, _, _ = hdt.hdt_add_norm_fwd(x, w, b, 0.0, y=y)
    # y is normalised up to its own roundings and the mean's: a few units of 2^-24 times the width's root
    assert float((h - wh).abs().max()) <= 64 * 2 ** -24 * float(wh.abs().max()) and float((n - want).abs().max()) <= 256 * 2 ** -24 * float(want.abs().max())


def test_nothing_is_written_behind_the_last_row():
    import torch
    import paper_2407_08330_amd as hdt
    for rows, width in ((3, 17), (5, 768), (2, 3001)):
        for dtype in (torch.bfloat16, torch.float32):
            def room(n, dt):
                t = torch.full((n + 64,), 7.0, dtype=dt, device="cuda")
                return t, t[:n]
            x, y, dn = (torch.randn(rows, width, device="cuda").to(dtype) for _ in range(3))
            w = torch.ones(width, device="cuda")
            big, small, st = [room(rows * width, dtype) for _ in range(4)], [room(width, torch.float32) for _ in range(5)], room(4 * rows, torch.float32)
            n, h, s = hdt.hdt_gate_norm_fwd(x, y, w, w, gate=w, post_bias=w, bias=w, h=big[0][1].view(rows, width), n=big[1][1].view(rows, width), stats=st[1].view(4, rows))
            hdt.hdt_gate_norm_bwd(dn, h, y, s, w, w, gate=w, post_bias=w, bias=True, dx=big[2][1].view(rows, width), dy=big[3][1].view(rows, width),
                                  **{k: v[1] for k, v in zip(GRADS[2:], small)})
            assert all(bool((r[len(v):] == 7).all()) and not bool((v == 7).all()) for r, v in (*big, *small, st))


def test_shapes_with_leading_dimensions_and_no_rows():
    import torch
    import paper_2407_08330_amd as hdt
    x, y, w = torch.randn(2, 3, 40, device="cuda"), torch.randn(2, 3, 40, device="cuda"), torch.randn(40, device="cuda")
    n, h, s = hdt.hdt_gate_norm_fwd(x, y, w, w)
    flat = hdt.hdt_gate_norm_fwd(x.view(6, 40), y.view(6, 40), w, w)
    assert s.shape == (4, 2, 3) and torch.equal(n.view(6, 40), flat[0]) and torch.equal(s.view(4, 6), flat[2])
    assert hdt.hdt_gate_norm_fwd(x[0, 0], y[0, 0], w, w)[2].shape == (4,)
    e, nan = torch.empty(0, 40, device="cuda"), torch.full_like(w, float("nan"))
    n, h, s = hdt.hdt_gate_norm_fwd(e, e, w, w, gate=w, post_bias=w)
    got = hdt.hdt_gate_norm_bwd(e, h, e, s, w, w, gate=w, post_bias=w, bias=True, **{k: nan.clone() for k in GRADS[2:]})
    assert n.shape == e.shape and s.shape == (4, 0) and all(bool((g == 0).all()) for g in got[2:])


def test_non_finite_rows_stay_alone():
    import torch
    import paper_2407_08330_amd as hdt
    for rms in (False, True):
        x, y, dn, w = *(torch.randn(9, 700, device="cuda") for _ in range(3)), torch.randn(700, device="cuda")
        want = hdt.hdt_gate_norm_fwd(x, y, w, w, gate=w, rms=rms)
        grads = hdt.hdt_gate_norm_bwd(dn, want[1], y, want[2], w, w, gate=w, dh=x, rms=rms)
        x, y, dn = x.clone(), y.clone(), dn.clone()
        x[1, 5], y[4, 6], dn[7, 8] = float("nan"), float("nan"), float("nan")
        got = hdt.hdt_gate_norm_fwd(x, y, w, w, gate=w, rms=rms)
        good = [0, 2, 3, 5, 6, 7, 8]
        assert torch.equal(got[0][good], want[0][good]) and torch.equal(got[1][good], want[1][good]) and bool(got[0][[1, 4]].isnan().all())
        back = hdt.hdt_gate_norm_bwd(dn, got[1], y, got[2], w, w, gate=w, dh=x, rms=rms)
        good = [0, 2, 3, 5, 6, 8]
        assert all(torch.equal(a[good], b[good]) and bool(a[[1, 4, 7]].isnan().all()) for a, b in zip(back[:2], grads[:2]))


def test_the_same_bits_every_time_captured_and_on_another_stream():
    import torch
    import paper_2407_08330_amd as hdt
    x, y, dn = (torch.randn(3000, 768, device="cuda").bfloat16() for _ in range(3))
    w = torch.randn(768, device="cuda")
    ws = torch.empty(hdt.load_library().hdt_gate_norm_bwd_workspace_bytes(3000, 768), dtype=torch.uint8, device="cuda")

    def step(back={}, **kw):
        n, h, s = hdt.hdt_gate_norm_fwd(x, y, w, w, gate=w, post_bias=w, bias=w, scale=0.5, **kw)
        return (n, h, s, *hdt.hdt_gate_norm_bwd(dn, h, y, s, w, w, gate=w, post_bias=w, bias=True, dh=x, scale=0.5, **back, **kw))

    want = step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):  # two graphs that share a workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(dict(workspace=ws)))
        graphs.append(graph)
    for r in range(3):
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(float("nan"))
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


def test_large():
    """More than 2^32 elements and more rows than a launch has workgroups."""
    import torch
    import paper_2407_08330_amd as hdt
    rows, width = 5_000_000, 880
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, width, device="cuda")
    w = torch.ones(width, device="cuda")
    n, h, s = hdt.hdt_gate_norm_fwd(x, x, w, w, gate=w)
    want = hdt.hdt_gate_norm_fwd(x[-3:].clone(), x[-3:].clone(), w, w, gate=w)
    assert torch.equal(n[-3:], want[0]) and torch.equal(h[-3:], want[1]) and torch.equal(s[:, -3:], want[2]) and not bool(n[:-3].any())
    del n
    dx, dy, *_ = hdt.hdt_gate_norm_bwd(x, h, x, s, w, w, gate=w)
    back = hdt.hdt_gate_norm_bwd(x[-3:].clone(), want[1], x[-3:].clone(), want[2], w, w, gate=w)
    assert torch.equal(dx[-3:], back[0]) and torch.equal(dy[-3:], back[1])
