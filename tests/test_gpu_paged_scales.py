"""Attention over pages at scales of 0 and beside it, where scores times the scale are moderate and scores by themselves need not be."""
import pytest
import torch

from tests.paged_helpers import Paged, attend, check_attention

pytestmark = pytest.mark.gpu

KINDS = [(torch.float32, False), (torch.bfloat16, False), (torch.float32, True), (torch.bfloat16, True)]


def enlarge_keys(p, by):
    """Keys that were random numbers about 1, in the cache's type."""
    if p.is_e4m3:
        p.k_scale = p.k_scale * by
    else:
        p.k = p.k * by


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens", [([6], [40]), ([2, 1], [700, 0]), ([90], [37])])
@pytest.mark.parametrize("scale", [0.0, -0.0])
def test_a_scale_of_0_weighs_all_keys_alike(dtype, is_e4m3, new, lens, scale):
    """... however large the products that it takes away: beyond float32's range, and near its end."""
    for size in (1e19, 3e18):
        p = Paged(61, new, lens, 2, 64, 16, is_e4m3)
        enlarge_keys(p, size)
        q = (size * torch.randn((sum(new), 4, 64), generator=p.g)).to(dtype)
        out, lse = attend(p, q, scale=scale)
        check_attention(p, q, out, lse, scale=scale)


@pytest.mark.parametrize("dtype,is_e4m3", KINDS)
@pytest.mark.parametrize("new,lens", [([6], [40]), ([90], [37])])
@pytest.mark.parametrize("scale", [1e-38, -1e-38, 2.0 ** -127, 2.0 ** -140])
def test_scales_that_float32_hardly_holds(dtype, is_e4m3, new, lens, scale):
    p = Paged(62, new, lens, 2, 64, 16, is_e4m3)
    enlarge_keys(p, 1e18)
    q = (1e18 * torch.randn((sum(new), 4, 64), generator=p.g)).to(dtype)
    scale = torch.tensor(scale).item()                     # as float32 holds it
    out, lse = attend(p, q, scale=scale)
    check_attention(p, q, out, lse, scale=scale)
