"""Dropout and norm on more than 2^31 elements, and more rows than the norm's forward has workgroups for at once: elements behind those
borders against the generator in whole numbers, and rows against a small call."""
import pytest

import norm_reference as nr

pytestmark = pytest.mark.gpu

SEED, STEP, SITE, P = 0x1234567, 5, 9, 0.25
T = int(P * 65536 + 0.5)


def factor(element):
    word = nr.philox(element // 8, SITE, STEP, SEED)[element % 8 // 2]
    return 65536 / (65536 - T) if (word >> 16 * (element % 2) & 0xFFFF) >= T else 0.0


def rng():
    import torch
    return torch.tensor([SEED, STEP], device="cuda")


def test_dropout_beyond_31_bits():
    import torch
    import paper_2407_08330_amd as hdt
    n = 2 ** 32 + 2 ** 20 + 13          # the last elements lie beyond 2^32
    y = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    out = hdt.hdt_dropout_add(y, P, rng(), SITE)
    keep = torch.tensor(65536 / (65536 - T)).bfloat16()
    for first in (0, 2 ** 31 - 40, 2 ** 32 - 40, n - 61):
        got = out[first:first + 61].cpu()
        want = torch.tensor([factor(first + i) for i in range(min(61, n - first))])
        assert torch.equal(got, torch.where(want > 0, keep, torch.zeros((), dtype=torch.bfloat16))), first
    half = int((out == 0).sum(dtype=torch.int64))
    assert abs(half / n - P) < 1e-4      # 2^32 of them: six deviations are 4e-5
    assert hdt.hdt_dropout_add(y, P, rng(), SITE, out=y) is y and torch.equal(y[-4096:], out[-4096:])


def test_norm_beyond_31_bits():
    import torch
    import paper_2407_08330_amd as hdt
    rows, width = 2 ** 22 + 5, 513       # odd: a row's chunks take numbers of two blocks
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    y = torch.ones_like(x)
    w = torch.randn(width, device="cuda")
    last = slice(rows - 3, rows)
    x[last] = torch.randn(3, width, device="cuda").bfloat16()
    drop = dict(p=P, rng=rng(), site=SITE)
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(x, w, w, y=y, **drop)
    f = torch.tensor([[factor(r * width + c) for c in range(width)] for r in range(rows - 3, rows)], device="cuda")
    assert torch.equal(h[last], (x[last].float() + f).bfloat16())
    # half a step of n, and fp32 statistics of 513 values
    exact = x[last].double() + f.double()
    centred = exact - exact.mean(1, keepdim=True)
    want = centred / torch.sqrt((centred ** 2).mean(1, keepdim=True) + 1e-5)
    off = (n[last].double() - (want * w.double() + w.double())).abs()
    assert bool((off <= 2.0 ** -8 * (want * w + w).abs() + 1e-4 * (1 + want.abs()) * w.abs()).all())
    dn = y                               # any values
    dx, dy, dw, db = hdt.hdt_add_norm_bwd(dn, h, w, mean, rstd, **drop)
    small = hdt.hdt_add_norm_bwd(*(t[last].clone() for t in (dn, h)), w, *(t[last].clone() for t in (mean, rstd)))
    assert torch.equal(dx[last], small[0])
    # dy is the unrounded gradient times the factor: half a step of each of the two roundings
    assert bool(((dy[last].float() - dx[last].float() * f).abs() <= 2.0 ** -7 * (dx[last].float() * f).abs()).all())
    assert bool(((dy[last] == 0) | (f > 0)).all()) and bool(torch.isfinite(dw).all())
    assert torch.equal(db, torch.full_like(db, float(rows)))  # sums of ones, exact in fp32 below 2^24
