"""CPU checks of the 64-bit reference the relative-bias attention is compared with: its gradients against central differences, its
buckets against the formula, and equality with plain softmax attention where the bias is nothing."""
import math

import numpy as np
import pytest

from rel_reference import Reference, t5_table


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_against_differences(causal):
    rng = np.random.default_rng(5)
    B, H, KV, n, D = 2, 2, 1, 9, 4
    lengths, table = [9, 6], t5_table(8, 6, not causal)
    x = [rng.normal(size=s) for s in ((B, H, n, D), (B, KV, n, D), (B, KV, n, D), (8, H))]
    d_o = rng.normal(size=(B, H, n, D))
    ref = Reference(*x, table, 0.5, causal, lengths, d_o=d_o, dtype="f32")

    def loss(y):
        return (Reference(*y, table, 0.5, causal, lengths, dtype="f32").o * d_o).sum()

    for which, name in enumerate(("dq", "dk", "dv", "dbias")):
        grad = getattr(ref, name)
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in grad.shape)
            up, down = [y.copy() for y in x], [y.copy() for y in x]
            up[which][at] += 1e-5
            down[which][at] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - grad[at]) <= 1e-8 * (1 + abs(grad).max())


@pytest.mark.parametrize("buckets,distance,both", [(32, 128, False), (32, 128, True), (64, 512, False), (16, 40, True), (2, 5, False), (4, 3, True)])
def test_buckets_are_the_formula(buckets, distance, both):
    table = t5_table(buckets, distance, both)
    half = buckets // 2 if both else buckets
    exact = half // 2
    for d in range(-distance, distance + 1):
        away = abs(d) if both else max(-d, 0)
        want = away
        if away >= exact:
            want = min(half - 1, exact + math.floor(math.log(away / exact) / math.log(distance / exact) * (half - exact) + 1e-9))
        assert table[d + distance] == want + (half if both and d > 0 else 0)
    assert table[0] == half - 1


def test_no_bias_is_plain_attention():
    rng = np.random.default_rng(6)
    q, k, v = (rng.normal(size=(1, 2, 7, 4)) for _ in range(3))
    ref = Reference(q, k, v, np.zeros((8, 2)), t5_table(8, 6, True), 0.3, False, dtype="f32")
    a = np.exp(np.einsum("bhid,bhjd->bhij", q, k) * 0.3)
    assert np.allclose(ref.o, a / a.sum(-1, keepdims=True) @ v, atol=1e-12)
    assert np.allclose(ref.lse, np.log(a.sum(-1)), atol=1e-12)
