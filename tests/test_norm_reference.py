"""CPU checks of the 64-bit reference of dropout and layer norm: the generator in two ways and by known vectors, the gradient by central
differences."""
import numpy as np

from norm_reference import backward, factors, forward, philox


def test_generator():
    assert philox(0, 0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox(0xFFFFFFFF, 0xFFFFFFFF, 0xFFFFFFFFFFFFFFFF, 0xFFFFFFFFFFFFFFFF) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    seed, step, site, p = 0x123456789ABCDEF0, 0x1111222233334444, 7, 0.3
    f, t = factors(45, p, seed, step, site), round(0.3 * 65536)
    for e in range(45):
        word = philox(e // 8, site, step, seed)[e % 8 // 2]
        u = word >> 16 if e % 2 else word & 0xFFFF
        assert f[e] == (65536 / (65536 - t) if u >= t else 0)


def test_share_that_is_kept():
    n, p = 200_000, 0.1
    f = factors(n, p, 5, 6, 7)
    assert abs((f == 0).mean() - p) <= 5 * np.sqrt(p * (1 - p) / n) + 1 / 65536
    assert abs(f.mean() - 1) <= 5 * np.sqrt(p / (1 - p) / n)


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    rows, width = 5, 7
    x, y, dn, dh = (rng.normal(size=(rows, width)) for _ in range(4))
    w, b, f = rng.normal(size=width), rng.normal(size=width), factors(rows * width, 0.25, 1, 2, 3).reshape(rows, width)

    def loss(x, y, w, b):
        out = forward(x, y, w, b, 1e-5, f, 0)
        return (out["n"][0] * dn).sum() + (out["h"][0] * dh).sum()

    out = forward(x, y, w, b, 1e-5, f, 0)
    grad = backward(dn, dh, out["h"][0], w, out["mean"][0], out["rstd"][0], f, 0, 0)
    for which, name in enumerate(("dx", "dy", "dw", "db")):
        for at in np.ndindex(grad[name][0].shape):
            step = [[v.copy() for v in (x, y, w, b)] for _ in range(2)]
            step[0][which][at] += 1e-6
            step[1][which][at] -= 1e-6
            assert abs((loss(*step[0]) - loss(*step[1])) / 2e-6 - grad[name][0][at]) <= 1e-7 * (1 + abs(grad[name][0]).max())
