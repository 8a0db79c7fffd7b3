"""Specs of rotary positions that say "all of the head" in different ways are the same spec, with a table too."""
import pytest
import torch

from paper_2607_02963_amd import pdec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_a_rotary_dim_of_0_is_the_whole_head(D):
    q = torch.randn((5, 3, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    pos = torch.arange(5, dtype=torch.int32, device="cuda") * 77
    freqs = 10000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device="cuda") / D)
    for kw in ({}, {"freqs": freqs}):
        want, _ = pdec.rope(q, None, pos, pdec.rope_spec(D, **kw))
        for R in (0, D):
            assert torch.equal(pdec.rope(q, None, pos, pdec.rope_spec(D, rotary_dim=R, **kw))[0], want)
    with pytest.raises(ValueError, match=f"{D // 2} elements"):
        pdec.rope_spec(D, rotary_dim=0, freqs=freqs[:0])
