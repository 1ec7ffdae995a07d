"""CPU checks of the strides that a call of the relative-bias attention is described by: every row that a description reaches lies in its
tensor.  A tensor without distance between its rows has none that the library takes (all three strides 0 stand for a dense one there)."""
import pytest


@pytest.fixture
def describe(monkeypatch):
    from paper_2407_08330_amd import binding, build
    import os
    if not os.path.exists(binding.library_path()):
        build.build()
    monkeypatch.setattr(binding, "_same_device", lambda ts: None)  # (the descriptions of host tensors are never run)

    def call(**kw):
        import torch
        t = dict(q=torch.zeros(2, 4, 8, 64), k=torch.zeros(2, 2, 9, 64), v=torch.zeros(2, 2, 9, 64))
        t.update(kw)
        return binding._rel_attn_call(t.pop("q"), t.pop("k"), t.pop("v"), torch.zeros(32, 4), torch.zeros(257, dtype=torch.int32), 0.125, True, None, None, **t)
    return call


NAMES = ["q", "k", "v", "o", "d_o", "dq", "dk", "dv"]


def shape_of(name):
    return (2, 2, 9, 64) if name in ("k", "v", "dk", "dv") else (2, 4, 8, 64)


@pytest.mark.parametrize("name", NAMES)
def test_one_row_for_all_is_refused(describe, name):
    import torch
    shape = shape_of(name)
    with pytest.raises(ValueError, match=f"{name}: .*row"):
        describe(**{name: torch.zeros(64).expand(shape)})
    with pytest.raises(ValueError, match=f"{name}: .*row"):
        describe(**{name: torch.zeros(shape[0], shape[1], 1, 64).expand(shape)})
    with pytest.raises(ValueError, match=f"{name}: .*row"):  # rows that reach into each other
        describe(**{name: torch.zeros(4096).as_strided(shape, (0, 0, 32, 1))})


def test_a_gradient_of_sums_is_refused(describe):
    """What autograd makes of (o.sum((0, 1, 2)) @ w).backward(): one row of 64 values with strides 0, 0, 0, 1."""
    import torch
    o = torch.zeros(2, 4, 8, 64, requires_grad=True)
    got = []
    o.register_hook(got.append)
    (o.sum((0, 1, 2)) @ torch.ones(64)).backward()
    assert got[0].stride() == (0, 0, 0, 1) and got[0].untyped_storage().nbytes() == 256
    with pytest.raises(ValueError, match="d_o"):
        describe(d_o=got[0])


@pytest.mark.parametrize("name", NAMES)
def test_descriptions_reach_nothing_but_the_tensor(describe, name):
    """Dense tensors, views, broadcasts over batch and heads, dimensions of one element with any stride."""
    import torch
    shape = shape_of(name)
    B, H, n, D = shape
    for t in (torch.zeros(shape), torch.zeros(B, n, H, D).transpose(1, 2), torch.zeros(1, 1, n, D).expand(shape), torch.zeros(1, H, n, D).expand(shape),
              torch.zeros(B, H, n, 2 * D)[..., D:], torch.zeros(B, 2 * H, 3 * n, D)[:, ::2, ::3]):
        c = getattr(describe(**{name: t}), name)
        s = (c.batch, c.head, c.row)
        if s == (0, 0, 0):
            assert t.is_contiguous()
            s = (H * n * D, n * D, D)
        assert s == t.stride()[:3]
    one = torch.zeros(64).expand(shape[:2] + (1, 64))  # one row a head, the same for all: no dense tensor
    call = dict(q=one, o=one) if name in ("q", "o", "d_o", "dq") else dict(k=one, v=one)
    if name in call:
        c = getattr(describe(**call), name)
        assert (c.batch, c.head, c.row) == (0, 0, 64)
