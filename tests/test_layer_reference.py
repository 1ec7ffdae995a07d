"""CPU checks of the 64-bit reference of embeddings, the gated feed-forward block and the norms around a block: gradients by central
differences."""
import numpy as np
import pytest

import layer_reference as lr


def check_gradients(loss, args, grads, which):
    for i, name in which:
        for at in np.ndindex(args[i].shape):
            step = [[a.copy() for a in args] for _ in range(2)]
            step[0][i][at] += 1e-6
            step[1][i][at] -= 1e-6
            assert abs((loss(*step[0]) - loss(*step[1])) / 2e-6 - grads[name][0][at]) <= 1e-7 * (1 + abs(grads[name][0]).max()), (name, at)


def test_embedding():
    rng = np.random.default_rng(1)
    ids, table, d = np.array([[3, 0, -1], [3, 7, 3]]), rng.normal(size=(5, 4)), rng.normal(size=(2, 3, 4))
    grad = {"dtable": lr.embed_grad(d, ids, 5, 1.5, 0)}
    check_gradients(lambda t: (lr.embed(ids, t, 1.5, 0)[0] * d).sum(), [table], grad, [(0, "dtable")])
    old = rng.normal(size=(5, 4))
    assert np.array_equal(lr.embed_grad(d, ids, 5, 1.5, 0, old)[0], grad["dtable"][0] + old)


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_feed_forward(name):
    rng = np.random.default_rng(2)
    x, wg, wu, wd, dy = (rng.normal(size=s) for s in ((3, 4), (5, 4), (5, 4), (4, 5), (3, 4)))

    def out(x, wg, wu, wd):
        return lr.ffn_out(lr.ffn_inner(x, wg, wu, name, 0)["hidden"][0], wd, 0)[0]

    kept = lr.ffn_inner(x, wg, wu, name, 0)
    grads = lr.ffn_grads(dy, x, wg, wu, wd, kept["by_gate"][0], kept["by_up"][0], kept["hidden"][0], 0)
    check_gradients(lambda *a: (out(*a) * dy).sum(), [x, wg, wu, wd], grads, list(enumerate(("dx", "dw_gate", "dw_up", "dw_down"))))
    if name != "silu":  # silu(1) = 1 / (1 + 1 / e), gelu(1) = Phi(1); the tanh's is within 0.001 of it
        assert abs(lr.act(np.array([1.0]), name)[0][0] - 0.8413447) <= (1e-7 if name == "gelu" else 1e-3)


@pytest.mark.parametrize("rms", [False, True])
def test_norms_around_a_block(rms):
    rng = np.random.default_rng(3)
    x, y, dn, dh = (rng.normal(size=(4, 6)) for _ in range(4))
    vectors = [rng.normal(size=6) for _ in range(5)]

    def loss(x, y, wp, bp, gate, w, b):
        out = lr.gate_norm(x, y, wp, bp, gate, w, b, 0.7, 1e-3, rms, 0)
        return (out["n"][0] * dn).sum() + (out["h"][0] * dh).sum()

    wp, bp, gate, w, b = vectors
    out = lr.gate_norm(x, y, wp, bp, gate, w, b, 0.7, 1e-3, rms, 0)
    grads = lr.gate_norm_grads(dn, dh, out["h"][0], y, out["stats"][0], wp, bp, gate, w, 0.7, rms, 0, 0)
    check_gradients(loss, [x, y, *vectors], grads, list(enumerate(("dx", "dy", "dpost_weight", "dpost_bias", "dgate", "dweight", "dbias"))))
