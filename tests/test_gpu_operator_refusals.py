"""Calls of relative-bias attention, dropout and norm that are refused before anything is launched, in the native and the general form:
tensors whose memory is smaller than their shape, numbers that do not fit."""
import pytest

from test_gpu_operator_binding import hdt, tensors  # noqa: F401  (hdt: a fixture, both forms)

pytestmark = pytest.mark.gpu


@pytest.fixture
def attention(hdt):  # noqa: F811
    import torch
    t = tensors(torch.float32)
    table = hdt.hdt_rel_table(32, 128)
    fwd = dict(q=t["q"], k=t["k"], v=t["v"], bias=t["bias"], table=table, softmax_scale=0.125)
    o, lse = hdt.hdt_rel_attn_fwd(**fwd)
    return fwd, dict(fwd, o=o, lse=lse, d_o=t["d_o"])


@pytest.mark.parametrize("name", ["q", "k", "v", "o", "d_o", "dq", "dk", "dv"])
def test_one_row_expanded_over_all(hdt, attention, name):  # noqa: F811
    """64 values in memory, a tensor of all the rows: as an input it would be read beyond its end, as a result written."""
    import torch
    fwd, bwd = attention
    shape = (fwd["k"] if name in ("k", "v", "dk", "dv") else fwd["q"]).shape
    row = torch.zeros(64, device="cuda").expand(shape)
    assert row.stride() == (0, 0, 0, 1)
    if name in ("q", "k", "v", "o"):
        with pytest.raises(ValueError, match=name):
            hdt.hdt_rel_attn_fwd(**{**fwd, name: row})
    with pytest.raises(ValueError, match=name):
        hdt.hdt_rel_attn_bwd(**{**bwd, name: row})


def test_sites_outside_32_bits(hdt):  # noqa: F811
    import torch
    t = tensors(torch.float32)
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"], p=0.1, rng=t["rng"], site=2 ** 32 - 1)
    for site in (-1, 2 ** 32, 2 ** 32 + 3, 2 ** 70):
        for call in (lambda: hdt.hdt_dropout_add(t["y"], 0.1, t["rng"], site), lambda: hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"], p=0.1, rng=t["rng"], site=site),
                     lambda: hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, p=0.1, rng=t["rng"], site=site)):
            with pytest.raises(ValueError, match="site"):
                call()


def test_workspaces_that_are_not_contiguous(hdt, attention):  # noqa: F811
    """A byte expanded to any size, and every second byte of a buffer: refused, however large they say they are."""
    import torch
    fwd, bwd = attention
    t = tensors(torch.float32)
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"], p=0.1, rng=t["rng"])
    for w in (torch.zeros(16, dtype=torch.uint8, device="cuda")[:1].expand(1 << 30), torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")[::2]):
        for call in (lambda: hdt.hdt_rel_attn_fwd(**fwd, workspace=w), lambda: hdt.hdt_rel_attn_bwd(**bwd, workspace=w),
                     lambda: hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, p=0.1, rng=t["rng"], workspace=w)):
            with pytest.raises(ValueError, match="workspace"):
                call()
