"""fbsr_round_i8 where a row has nothing in it."""
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
