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
