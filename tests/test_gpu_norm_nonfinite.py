"""Dropout and norm on NaN and infinities: they stay in their row (and in the sums over rows that they go into)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("name", ["bfloat16", "float32"])
@pytest.mark.parametrize("width", [8, 77, 768, 2049, 8200])
def test_norm(width, name, value):
    import torch
    import paper_2407_08330_amd as hdt
    rows, row, col = 9, 4, width // 2
    x, y, dn, dh = (torch.randn(rows, width, device="cuda").to(getattr(torch, name)) for _ in range(4))
    w = torch.randn(width, device="cuda")
    rng = torch.tensor([1, 2], device="cuda")
    other = torch.arange(rows, device="cuda") != row
    for p in (0.0, 0.5):
        kw = dict(p=p, rng=rng, site=3)
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w, w, y=y, **kw)
        dx, dy, dw, db = hdt.hdt_add_norm_bwd(dn, h, w, mean, rstd, dh=dh, **kw)
        for which in ("x", "y"):
            t = dict(x=x.clone(), y=y.clone())
            t[which][row, col] = value
            n2, h2, mean2, rstd2 = hdt.hdt_add_norm_fwd(t["x"], w, w, y=t["y"], **kw)
            assert bool(torch.isnan(n2[row]).all()) and not bool(torch.isfinite(mean2[row])) and not bool(torch.isfinite(h2[row, col]))
            assert all(torch.equal(a[other], b[other]) for a, b in zip((n, h, mean, rstd), (n2, h2, mean2, rstd2)))
            g = hdt.hdt_add_norm_bwd(dn, h2, w, mean2, rstd2, dh=dh, **kw)
            assert bool(torch.isnan(g[0][row]).all()) and bool(torch.isnan(g[2]).all()) and torch.equal(g[3], db)
            assert torch.equal(g[0][other], dx[other]) and torch.equal(g[1][other], dy[other])
        dn2 = dn.clone()
        dn2[row, col] = value
        g = hdt.hdt_add_norm_bwd(dn2, h, w, mean, rstd, dh=dh, **kw)
        assert not bool(torch.isfinite(g[0][row]).any()) and torch.equal(g[0][other], dx[other]) and torch.equal(g[1][other], dy[other])
        rest = torch.arange(width, device="cuda") != col
        assert not bool(torch.isfinite(g[2][col])) and not bool(torch.isfinite(g[3][col]))
        assert torch.equal(g[2][rest], dw[rest]) and torch.equal(g[3][rest], db[rest])


@pytest.mark.parametrize("name", ["bfloat16", "float32"])
def test_dropout(name):
    import torch
    import paper_2407_08330_amd as hdt
    y, x = (torch.randn(5003, device="cuda").to(getattr(torch, name)) for _ in range(2))
    rng = torch.tensor([1, 2], device="cuda")
    want = hdt.hdt_dropout_add(y, 0.5, rng, x=x)
    at = torch.arange(0, 5003, 97, device="cuda")
    for value in (float("nan"), float("inf")):
        bad = y.clone()
        bad[at] = value
        got = hdt.hdt_dropout_add(bad, 0.5, rng, x=x)
        assert not bool(torch.isfinite(got[at]).any())     # 0 times either is a NaN
        got[at] = want[at]
        assert torch.equal(got, want)
