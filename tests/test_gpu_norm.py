"""GPU tests of dropout, residual and layer norm against the 64-bit reference (tests/norm_reference.py), each output within the bound of its
own roundings; masks element by element."""
import numpy as np
import pytest

import norm_reference as nr
from gpu_common import GuardedWorkspace, from_dev, say
from rel_reference import check, half_step
from test_gpu_rel_attn import dev, values

pytestmark = pytest.mark.gpu

SEED, STEP = -0x123456789ABCDEF, 0x7000000012345678   # all 64 bits count, the sign too


def rng_tensor(seed=SEED, step=STEP):
    import torch
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


def factors(shape, p, site):
    return nr.factors(int(np.prod(shape)), p, SEED & (2 ** 64 - 1), STEP, site).reshape(shape)


def host(t):
    return from_dev(t).astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 65535 / 65536, 1e-6])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 2049, 100_003])
def test_dropout_add(n, p, dtype):
    import torch
    import paper_2407_08330_amd as hdt
    gen = np.random.default_rng(n)
    y, x = values(gen, (n,), dtype), values(gen, (n,), dtype)
    f = factors((n,), p, 11)
    for residual in (None, x):
        want, bound = nr.dropout_add(y, residual, f, half_step(dtype))
        out = torch.full((n + 24,), 7.0, dtype=dev(y, dtype).dtype, device="cuda")
        hdt.hdt_dropout_add(dev(y, dtype), p, rng_tensor(), site=11, x=None if residual is None else dev(residual, dtype), out=out[:n])
        check(host(out[:n]), want, bound, f"n={n} p={p}")
        assert bool((out[n:] == 7).all())


def test_dropout_in_place_and_its_gradient():
    import torch
    import paper_2407_08330_amd as hdt
    y = torch.randn(5000, device="cuda")
    x = torch.randn_like(y)
    want = hdt.hdt_dropout_add(y, 0.3, rng_tensor(), 4, x=x)
    assert torch.equal(hdt.hdt_dropout_add(y, 0.3, rng_tensor(), 4, x=x, out=y), want)
    y = torch.ones(5000, device="cuda")
    kept = hdt.hdt_dropout_add(y, 0.3, rng_tensor(), 4)
    g = torch.randn_like(y)
    assert torch.equal(hdt.hdt_dropout_add(g, 0.3, rng_tensor(), 4), g * kept)
    for other in (hdt.hdt_dropout_add(y, 0.3, rng_tensor(), 5), hdt.hdt_dropout_add(y, 0.3, rng_tensor(step=STEP + 1), 4),
                  hdt.hdt_dropout_add(y, 0.3, rng_tensor(step=STEP ^ (1 << 40)), 4), hdt.hdt_dropout_add(y, 0.3, rng_tensor(seed=SEED ^ (1 << 50)), 4)):
        assert 0.5 < float((other == kept).float().mean()) < 0.66  # 0.58 for masks that have nothing to do with each other


ROWS = [(1, 1), (1, 768), (4, 768), (5, 7), (3, 8), (9, 9), (130, 1000), (7, 511), (6, 513), (300, 64), (2, 1024), (3, 1025), (5, 2048), (2, 2049), (3, 8192),
        (2, 8193), (2, 32768), (2, 32761), (4100, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", ROWS)
def test_add_norm(rows, width, dtype):
    import paper_2407_08330_amd as hdt
    say(f"[norm] {rows} x {width} {dtype}")
    gen = np.random.default_rng(rows * 40000 + width)
    u = half_step(dtype)
    for p, with_y, with_bias, with_dh, wdt in ((0.1, True, True, True, dtype), (0.0, True, False, False, "f32"), (0.0, False, True, True, "bf16"),
                                               (0.25, True, True, False, dtype)):
        x, y, dn, dh = (values(gen, (rows, width), dtype) for _ in range(4))
        x = x + 3
        w, b = 1 + values(gen, (width,), wdt) / 4, values(gen, (width,), wdt)
        x, w = (host(dev(inexact, d)) for inexact, d in ((as_type(x, dtype), dtype), (as_type(w, wdt), wdt)))
        f = factors((rows, width), p, 2 ** 32 - 1)
        want = nr.forward(x, y if with_y else None, w, b if with_bias else None, 1e-5, f, u)
        drop = dict(p=p, rng=rng_tensor(), site=2 ** 32 - 1)
        dx_, dy_, dw_, db_ = (dev(t, d) for t, d in ((x, dtype), (y, dtype), (w, wdt), (b, wdt)))
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(dx_, dw_, db_ if with_bias else None, 1e-5, y=dy_ if with_y else None, **drop)
        assert with_y or h is dx_
        for name, t in (("h", h), ("n", n), ("mean", mean), ("rstd", rstd)):
            if with_y or name != "h":
                check(host(t), *want[name], name)
        need = hdt.load_library().hdt_add_norm_bwd_workspace_bytes(rows, width)
        ws = GuardedWorkspace(need)
        got = hdt.hdt_add_norm_bwd(dev(dn, dtype), h, dw_, mean, rstd, dh=dev(dh, dtype) if with_dh else None, bias=with_bias, workspace=ws.view,
                                   **(drop if with_y else {}))
        ws.check()
        want = nr.backward(dn, dh if with_dh else None, host(h), w, host(mean), host(rstd), f if with_y else np.ones_like(f), u, half_step(wdt))
        assert (got[1] is got[0]) == (p == 0 or not with_y) and (got[3] is not None) == with_bias
        for name, t in zip(("dx", "dy", "dw", "db"), got):
            if t is not None:
                check(host(t), *want[name], name)


def as_type(x, dtype):
    from paper_2407_08330_amd import inputs
    return inputs.round_to_bf16(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float32)


def test_nothing_is_written_behind_the_last_row():
    import torch
    import paper_2407_08330_amd as hdt
    for rows, width in ((3, 17), (5, 768), (2, 3001)):
        for dtype in (torch.bfloat16, torch.float32):
            def room():
                t = torch.full((rows * width + 64,), 7.0, dtype=dtype, device="cuda")
                return t, t[:rows * width].view(rows, width)
            x, y, dn = (torch.randn(rows, width, device="cuda").to(dtype) for _ in range(3))
            w = torch.ones(width, device="cuda")
            bufs = [room() for _ in range(4)]
            n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w, w, y=y, p=0.2, rng=rng_tensor(), h=bufs[0][1], n=bufs[1][1])
            hdt.hdt_add_norm_bwd(dn, h, w, mean, rstd, p=0.2, rng=rng_tensor(), dx=bufs[2][1], dy=bufs[3][1])
            assert all(bool((b[rows * width:] == 7).all()) and not bool((v == 7).all()) for b, v in bufs)


def test_shapes_with_leading_dimensions_and_no_rows():
    import torch
    import paper_2407_08330_amd as hdt
    x, w = torch.randn(2, 3, 40, device="cuda"), torch.randn(40, device="cuda")
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w)
    flat = hdt.hdt_add_norm_fwd(x.view(6, 40), w)
    assert h is x and mean.shape == (2, 3) and torch.equal(n.view(6, 40), flat[0]) and torch.equal(rstd.view(6), flat[3])
    e = torch.empty(0, 40, device="cuda")
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(e, w, y=e, p=0.5, rng=rng_tensor())
    dx, dy, dw, db = hdt.hdt_add_norm_bwd(e, h, w, mean, rstd, p=0.5, rng=rng_tensor(), dweight=torch.full_like(w, float("nan")), dbias=torch.full_like(w, float("nan")))
    assert n.shape == e.shape and bool((dw == 0).all()) and bool((db == 0).all())


def test_the_same_bits_every_time():
    import torch
    import paper_2407_08330_amd as hdt
    x, y, dn = (torch.randn(5000, 768, device="cuda").bfloat16() for _ in range(3))
    w = torch.randn(768, device="cuda")
    drop = dict(p=0.1, rng=rng_tensor(), site=1)
    first = None
    for _ in range(4):
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w, y=y, **drop)
        got = (n, h, mean, rstd, *hdt.hdt_add_norm_bwd(dn, h, w, mean, rstd, dh=y, **drop))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_captured_with_a_step_that_moves():
    """A graph of forward and backward that counts its own step up: every replay drops what an eager pass of that step drops."""
    import torch
    import paper_2407_08330_amd as hdt
    x, y, dn = (torch.randn(64, 200, device="cuda") for _ in range(3))
    w = torch.randn(200, device="cuda")
    state = rng_tensor(step=40)
    ws = torch.empty(hdt.load_library().hdt_add_norm_bwd_workspace_bytes(64, 200), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(x) for _ in range(5)] + [torch.empty(64, device="cuda") for _ in range(2)] + [torch.empty_like(w) for _ in range(2)]

    def step(rng):
        hdt.hdt_dropout_add(y, 0.5, rng, 1, out=out[4])
        hdt.hdt_add_norm_fwd(x, w, w, y=y, p=0.5, rng=rng, site=2, h=out[0], n=out[1], mean=out[5], rstd=out[6])
        hdt.hdt_add_norm_bwd(dn, out[0], w, out[5], out[6], p=0.5, rng=rng, site=2, dx=out[2], dy=out[3], dweight=out[7], dbias=out[8], workspace=ws)

    step(state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(state)
        state[1].add_(1)
    seen = []
    for r in range(4):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        step(rng_tensor(step=40 + r))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out)), f"replay {r}"
        seen.append(got[4])
    assert not any(torch.equal(seen[0], t) for t in seen[1:])


def test_on_another_stream():
    import torch
    import paper_2407_08330_amd as hdt
    from gpu_common import busy
    x, y, dn = (torch.randn(300, 768, device="cuda").bfloat16() for _ in range(3))
    w = torch.randn(768, device="cuda")
    drop = dict(p=0.1, rng=rng_tensor(), site=1)

    def run(**kw):
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w, y=y, **drop, **kw)
        return (n, h, *hdt.hdt_add_norm_bwd(dn, h, w, mean, rstd, **drop, **kw), hdt.hdt_dropout_add(x, stream=kw.get("stream"), **drop))

    want = run()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    got = run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
