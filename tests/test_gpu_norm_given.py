"""Tensors that a caller gives for the norm's results are written in every form of the call, also where a result is a copy: the gradient of
y where nothing is dropped, h where there is no y."""
import pytest

from test_gpu_operator_binding import hdt  # noqa: F401  (a fixture, both forms)

pytestmark = pytest.mark.gpu


def tensors(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    n = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    return dict(x=n(50, 77), y=n(50, 77), dn=n(50, 77), dh=n(50, 77), w=n(77), b=n(77))


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
@pytest.mark.parametrize("p", [0.0, 1e-6])   # the second rounds to nothing in steps of 1 / 65536
def test_the_gradient_of_y_where_nothing_is_dropped(hdt, p, name):  # noqa: F811
    import torch
    t = tensors(getattr(torch, name))
    rng = torch.tensor([1, 2], device="cuda")
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], y=t["y"], p=p, rng=rng)
    want = hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dh=t["dh"], p=p, rng=rng)
    assert want[1] is want[0]
    for side in (None, torch.cuda.Stream()):
        dy = torch.full_like(t["x"], 7.0)
        torch.cuda.synchronize()
        got = hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dh=t["dh"], p=p, rng=rng, dy=dy, stream=side)
        torch.cuda.synchronize()
        assert got[1] is dy and got[0] is not dy
        assert torch.equal(dy, want[0]) and all(torch.equal(a, b) for a, b in zip(got, want))
    both = torch.empty_like(t["x"])
    got = hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dh=t["dh"], p=p, rng=rng, dx=both, dy=both)
    assert got[0] is both and got[1] is both and torch.equal(both, want[0])
    for other in (h, t["dn"], t["dh"]):
        before = other.clone()
        with pytest.raises(ValueError):
            hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dh=t["dh"], p=p, rng=rng, dy=other)
        assert torch.equal(other, before)
    with pytest.raises(ValueError):
        hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, p=p, rng=rng, dy=torch.empty(50, 78, device="cuda", dtype=h.dtype))


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_h_without_y(hdt, name):  # noqa: F811
    import torch
    t = tensors(getattr(torch, name))
    want = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"])
    assert want[1] is t["x"]
    for side in (None, torch.cuda.Stream()):
        h = torch.full_like(t["x"], 7.0)
        torch.cuda.synchronize()
        got = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], h=h, stream=side)
        torch.cuda.synchronize()
        assert got[1] is h and all(torch.equal(a, b) for a, b in zip(got, want))
    got = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], h=t["x"])
    assert got[1] is t["x"] and torch.equal(got[0], want[0])
    n = torch.empty_like(t["x"])
    with pytest.raises(ValueError):
        hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], h=n, n=n)


def test_no_rows(hdt):  # noqa: F811
    import torch
    e, w = torch.empty(0, 16, device="cuda"), torch.ones(16, device="cuda")
    h, dy = torch.empty_like(e), torch.empty_like(e)
    n, h2, mean, rstd = hdt.hdt_add_norm_fwd(e, w, h=h)
    assert h2 is h
    assert hdt.hdt_add_norm_bwd(e, h, w, mean, rstd, dy=dy)[1] is dy


def test_captured_where_nothing_is_dropped(hdt):  # noqa: F811
    """A step into the program's own buffers, replayed with new values: every buffer holds what an eager step gives."""
    import torch
    t = tensors(torch.float32)
    out = dict(h=torch.empty_like(t["x"]), dx=torch.empty_like(t["x"]), dy=torch.empty_like(t["x"]), h1=torch.empty_like(t["x"]))
    ws = torch.empty(hdt.load_library().hdt_add_norm_bwd_workspace_bytes(50, 77), dtype=torch.uint8, device="cuda")

    def step():
        hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], h=out["h1"])
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], y=t["y"], h=out["h"])
        hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dx=out["dx"], dy=out["dy"], workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(4):
        for k in ("x", "y", "dn"):
            t[k].copy_(torch.randn_like(t[k]))
        for v in out.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], out[k]) for k in out), f"replay {r}"
        assert torch.equal(got["dy"], got["dx"]) and torch.equal(got["h1"], t["x"])
