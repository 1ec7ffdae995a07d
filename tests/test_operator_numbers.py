"""CPU checks of numbers that the binding of dropout, norm and relative-bias attention does not pass on cut to 32 bits."""
import os

import pytest


@pytest.fixture
def hdt():
    import paper_2407_08330_amd as hdt
    from paper_2407_08330_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build()
    return hdt


@pytest.mark.parametrize("site", [-1, 2 ** 32, 2 ** 32 + 3, -2 ** 40])
def test_sites_outside_32_bits(hdt, site):
    import torch
    x, w, rng, one = torch.zeros(2, 8), torch.zeros(8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    for call in (lambda: hdt.hdt_dropout_add(x, 0.1, rng, site), lambda: hdt.hdt_add_norm_fwd(x, w, w, y=x, p=0.1, rng=rng, site=site),
                 lambda: hdt.hdt_add_norm_bwd(x, x, w, one, one, p=0.1, rng=rng, site=site)):
        with pytest.raises(ValueError, match="site"):
            call()


@pytest.mark.parametrize("buckets,distance", [(2 ** 32 + 32, 128), (32, 2 ** 32 + 128), (-2 ** 32 + 32, 128), (2 ** 31, 128), (32, -2 ** 33 + 128)])
def test_tables_of_more_than_32_bits(hdt, buckets, distance, monkeypatch):
    """Refused by their numbers, before memory is asked for."""
    import torch
    from paper_2407_08330_amd import binding
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: pytest.fail("memory was asked for"))
    with pytest.raises(ValueError, match="32 bits"):
        binding.hdt_rel_table(buckets, distance, device="cpu")


def test_sizes_of_more_than_32_bits(hdt, monkeypatch):
    """Shapes that only an expanded or an empty tensor has here."""
    import torch
    from paper_2407_08330_amd import binding
    monkeypatch.setattr(binding, "_same_device", lambda ts: None)
    many = 2 ** 32 + 4
    q, k = torch.zeros(1, 4, 8, 64), torch.zeros(1, 4, 8, 64)
    bias, table = torch.zeros(32, 4), torch.zeros(257, dtype=torch.int32)

    def describe(q, k, bias):
        return binding._rel_attn_call(q, k, k, bias, table, 0.125, True, None, None)
    describe(q, k, bias)
    for bad in (dict(k=k[:, :1].expand(1, many, 8, 64)), dict(q=q.expand(many, 4, 8, 64), k=k.expand(many, 4, 8, 64))):
        with pytest.raises(ValueError, match="32 bits"):
            describe(**{**dict(q=q, k=k, bias=bias), **bad})
    x = torch.zeros(0, 2 ** 32 + 8)
    with pytest.raises(ValueError, match="32 bits"):
        binding._check_norm(x, torch.zeros(0), (), ())
