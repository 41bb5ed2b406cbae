"""fbsr_round_i8 where a row has nothing in it, and the signs of its zeros."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    module.fbsr = fbsr


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_without_columns_have_the_smallest_scale(src):
    """No element: the largest magnitude is 0, so the scale is 2^-126, in memory that held something else too."""
    x = torch.empty(37, 0, dtype=src, device="cuda")
    for scales in (None, torch.full((37,), 9.0, device="cuda")):
        codes, got = fbsr.fbsr_round_i8(x, "srf", 4, 1, scales=scales, values=torch.empty_like(x) if scales is None else None)
        assert codes.shape == (37, 0) and (scales is None or got is scales)
        assert bool((got == 2.0 ** -126).all())
    room = torch.full((37,), 7.0, device="cuda")
    fbsr.fbsr_round_i8(x[:12], "rtne", 1, 0, scales=room[:12])
    assert bool((room[:12] == 2.0 ** -126).all() and (room[12:] == 7).all())


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("variant,k", [("srff", 4), ("srf", 4), ("srf", 16), ("src", 3), ("src", 16), ("rtne", 1), ("rta", 1), ("rto", 1)])
def test_values_are_codes_times_scales_to_the_bit(variant, k, src):
    """An integer has one zero, so a negative element that is rounded to it reads as +0, whatever the variant."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for cols in (40, 700, 5000, 17000):
        x = torch.randn(6, cols, device="cuda", generator=gen) * torch.exp2(-6 * torch.rand(6, cols, device="cuda", generator=gen))
        x[0] = -0.0
        x[1, 5], x[2, 7] = float("-inf"), -0.0
        x = x.to(src)
        values = torch.full_like(x, 9.0)
        codes, scales = fbsr.fbsr_round_i8(x, variant, k, 1, values=values)
        assert int((codes[:, :cols][x < 0] == 0).sum()) > 0
        want = (codes[:, :cols].float() * scales[:, None]).to(src)
        bits = torch.int32 if src is torch.float32 else torch.int16
        assert torch.equal(values.view(bits), want.view(bits))
